"""Drafted trees on the GPU: layout, attention and acceptance against plain implementations (attention in 64 bits)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fa():
    from paper_2608_13667_amd import forkattn
    return forkattn


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def _i64(masks):
    return torch.from_numpy(np.asarray(masks, np.uint64).view(np.int64).copy()).cuda()


def _parents(rng, n, unused=0.1, back=6):
    used, out = [0], [-1]
    for i in range(1, n):
        if rng.random() < unused:
            out.append(-1)
        else:
            out.append(int(rng.choice(used[-back:])))
            used.append(i)
    return out


def _masks(parents):
    m = []
    for i, a in enumerate(parents):
        m.append(1 << i | (m[a] if 0 <= a < i else 0))
    return m


# ------------------------------------------------------------------------------------------------- layout

@pytest.mark.parametrize("N,n", [(1, 1), (1, 64), (5, 16), (7, 63), (513, 33)])
def test_layout(fa, N, n):
    rng = np.random.default_rng(N * 100 + n)
    trees = [_parents(rng, n) for _ in range(N - 1)] + [[-1] + list(range(n - 1))]  # the last one a chain
    base = rng.integers(0, 1 << 30, N)
    masks = torch.full((N, n), -7, dtype=torch.int64, device="cuda")
    pos = torch.full((N, n), -7, dtype=torch.int32, device="cuda")
    err = _i32([0])
    fa.tree_layout(_i32(trees), _i32(base), masks, pos, err=err)
    want = np.array([_masks(t) for t in trees], np.uint64)
    assert np.array_equal(masks.cpu().numpy().view(np.uint64), want)
    depth = np.array([[bin(int(x)).count("1") - 1 for x in row] for row in want])
    assert np.array_equal(pos.cpu().numpy(), base[:, None] + depth)
    assert int(err) == 0


def test_layout_flags_parents_that_are_not_before_their_node(fa):
    for bad, n in (([-1, 0, 2, 1], 4), ([-1, 0, 3, 1], 4), ([0, 0], 2), ([-2], 1), ([-1, 2**31 - 1, -2**31], 3)):
        masks, pos = torch.empty(2, n, dtype=torch.int64, device="cuda"), torch.empty(2, n, dtype=torch.int32, device="cuda")
        err = _i32([0])
        fa.tree_layout(_i32([[-1] * n, bad]), _i32([10, 20]), masks, pos, err=err)
        assert int(err) == fa.ERR_BAD_TREE
        good = [a if 0 <= a < i else -1 for i, a in enumerate(bad)]
        assert masks[1].tolist() == _masks(good) and masks[0].tolist() == [1 << i for i in range(n)]
        fa.tree_layout(_i32([[-1] * n, bad]), _i32([10, 20]), masks, pos)  # without a place for the flag


# ---------------------------------------------------------------------------------------------- attention

def _bf16(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).bfloat16()


class Tree:
    """Inputs of one call on the CPU, the 64-bit result, and the call."""

    def __init__(self, hq, hkv, d, n, prefix, suffix, masks, paged=False, seed=0, spare=3, scale=0.0, junk=float("nan")):
        rng = np.random.default_rng(seed)
        N = len(suffix)
        self.hq, self.hkv, self.d, self.N, self.n, self.prefix, self.suffix, self.paged = hq, hkv, d, N, n, prefix, suffix, paged
        self.scale, self.masks, self.cap = scale, masks, max(suffix) + n + spare
        self.q = _bf16(rng, N, n, hq, d)
        self.pk, self.pv = _bf16(rng, hkv, prefix, d), _bf16(rng, hkv, prefix, d)
        self.sk, self.sv = _bf16(rng, N, hkv, self.cap, d), _bf16(rng, N, hkv, self.cap, d)
        for b, length in enumerate(suffix):  # what is behind the nodes must not count
            self.sk[b, :, length + n:] = junk
            self.sv[b, :, length + n:] = junk
        self.rng = rng

    def want(self):
        """out, lse, and what a result may be off by: tolerances of each from the sums' sizes."""
        G, scale = self.hq // self.hkv, self.scale or 1 / math.sqrt(self.d)
        out = np.zeros((self.N, self.n, self.hq, self.d))
        lse = np.full((self.N, self.n, self.hq), -np.inf)
        tol, tol_lse = np.zeros_like(out), np.zeros_like(lse)
        to64 = lambda t: t.double().numpy()  # noqa: E731
        q, pk, pv, sk, sv = (to64(t) for t in (self.q, self.pk, self.pv, self.sk, self.sv))
        for b, length in enumerate(self.suffix):
            for i in range(self.n):
                see = list(range(length)) + [length + j for j in range(self.n) if int(self.masks[b][i]) >> j & 1]
                for h in range(self.hq):
                    g = h // G
                    k, v = np.concatenate([pk[g], sk[b, g, see]]), np.concatenate([pv[g], sv[b, g, see]])
                    if not len(k):
                        continue
                    with np.errstate(invalid="ignore"):
                        s = k @ q[b, i, h] * scale
                        m = s.max()
                        p = np.exp(s - m)
                        out[b, i, h] = p @ v / p.sum()
                        lse[b, i, h] = m + np.log(p.sum())
                        # a score: d exact products in steps of 32 and at most 32 roundings in each, relative to the sum of magnitudes,
                        # and the argument of the exponential; then the exponential.  p is rounded in two bf16 terms (2^-8 squared),
                        # the sums over keys take two steps for each 32 keys and a few in the merge.
                        size = (np.abs(k) @ np.abs(q[b, i, h])).max() * scale
                        rel = 2.0 ** -24 * (2 * ((32 + self.d / 32 + 8) * size + 4) + 2 * (len(k) / 16 + 64))
                        tol[b, i, h] = (p @ np.abs(v) / p.sum()) * (2.0 ** -16 + rel)
                        tol_lse[b, i, h] = rel + 2.0 ** -22 * abs(lse[b, i, h])
        return out, lse, tol, tol_lse

    def place(self):
        """The call's tensors on the GPU."""
        c = lambda t: t.cuda()  # noqa: E731
        self.lens, self.dmasks, self.dq = _i32(self.suffix), _i64(self.masks), c(self.q)
        self.out = torch.full((self.N, self.n, self.hq, self.d), float("nan"), device="cuda")
        self.lse = torch.full((self.N, self.n, self.hq), float("nan"), device="cuda")
        if not self.paged:
            self.cache = [c(t) for t in (self.pk, self.pv, self.sk, self.sv)]
            return
        shared, each = -(-self.prefix // 16), -(-self.cap // 16)
        pages = shared + self.N * each + 2
        ids = self.rng.permutation(pages)
        pools = []
        for pre, suf in ((self.pk, self.sk), (self.pv, self.sv)):
            pool = torch.full((pages, self.hkv, 16, self.d), float("nan"), dtype=torch.bfloat16)
            for i in range(self.prefix):
                pool[ids[i // 16], :, i % 16] = pre[:, i]
            for b in range(self.N):
                for u in range(self.cap):
                    pool[ids[shared + b * each + u // 16], :, u % 16] = suf[b, :, u]
            pools.append(c(pool))
        table = np.array([np.concatenate([ids[:shared], ids[shared + b * each: shared + (b + 1) * each]]) for b in range(self.N)])
        self.cache = pools + [_i32(table)]

    def plan(self, fa, max_len=None, blocks=0):
        top = self.cap if max_len is None else max_len
        if self.paged:
            return fa.Plan.tree_paged_plan(self.hq, self.hkv, self.d, self.N, self.n, self.prefix, self.cache[2].shape[1],
                                           self.cache[0].shape[0], top, softmax_scale=self.scale, blocks=blocks)
        return fa.Plan.tree_plan(self.hq, self.hkv, self.d, self.N, self.n, self.prefix, self.cap, top, softmax_scale=self.scale,
                                 blocks=blocks)

    def call(self, plan):
        attend = plan.tree_attend_paged if self.paged else plan.tree_attend
        attend(self.dq, *self.cache, self.lens, self.dmasks, self.out, self.lse)


def _close(t, want):
    out, lse, tol, tol_lse = want
    got, got_lse = t.out.double().cpu().numpy(), t.lse.double().cpu().numpy()
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got_lse), empty)
    assert (got[empty] == 0).all()
    assert (np.abs(got - out) <= tol).all(), f"worst {np.max(np.abs(got - out) / np.maximum(tol, 1e-300))} of the tolerance"
    assert (np.abs(got_lse[~empty] - lse[~empty]) <= tol_lse[~empty]).all()


def _trees(seed, N, n):
    rng = np.random.default_rng(seed)
    return [_masks(_parents(rng, n)) for _ in range(N)]


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("hq,hkv,d,n,prefix,suffix", [
    (8, 2, 64, 8, 70, [0, 5, 64, 17, 1]),
    (10, 2, 128, 16, 129, [0, 40, 7]),
    (4, 4, 128, 1, 200, [3, 0, 130]),        # nothing drafted, one query head per KV head
    (5, 1, 128, 64, 33, [9, 70]),            # the largest tree
    (7, 1, 64, 63, 0, [0, 1, 15, 16, 65]),   # no prefix
    (64, 1, 128, 3, 65, [31, 2]),            # a wide group
    (2, 2, 64, 13, 300, [700]),              # a long suffix
    (3, 3, 128, 1, 0, [0, 1]),               # the root alone
], ids=str)
def test_attend(fa, hq, hkv, d, n, prefix, suffix, paged):
    t = Tree(hq, hkv, d, n, prefix, suffix, _trees(n, len(suffix), n), paged, seed=n + prefix)
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    _close(t, t.want())
    assert plan.device_error() == 0


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
def test_attend_over_a_long_prefix(fa, paged):
    """Several ranges of whole tiles; the 64-bit result over one head's rows of a few nodes."""
    t = Tree(10, 2, 128, 9, 5000 + 13, [100, 0, 33], _trees(3, 3, 9), paged, seed=5)
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    _close(t, t.want())


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_many_rows_over_many_keys(fa, d, paged):
    """400 rows of a KV head over 8200 keys: the kernel in two phases to a tile, with two terms of p."""
    t = Tree(10, 2, d, 16, 8200 + 5, [100, 0, 33, 64, 7], _trees(5, 5, 16), paged, seed=d)
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    want = t.want()
    _close(t, want)
    first = t.out.clone()
    t.out.zero_()
    t.call(plan)
    assert torch.equal(first, t.out)


# few rows (two waves to a unit), a few units (tiles one after the other), many rows over many keys (two phases to a tile)
KINDS = [(8, 2, 3, 4, 300), (10, 2, 4, 12, 300), (10, 2, 5, 16, 8192)]


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("kind", KINDS, ids=["halves", "stream", "phases"])
def test_attend_infinite_prefix_values(fa, kind, paged):
    """In the prefix, which every row reads, an infinity stays in its channel and is that infinity; both signs, or a NaN, are NaN there."""
    hq, hkv, N, n, prefix = kind
    t = Tree(hq, hkv, 128, n, prefix, [5] * N, _trees(3, N, n), paged, seed=1)
    inf, nan = float("inf"), float("nan")
    t.pv[0, 17, 3], t.pv[0, prefix - 1, 9], t.pv[0, 200, 20], t.pv[0, 40, 20] = inf, -inf, inf, -inf
    t.pv[1, 250, 100], t.pv[1, 63, 64], t.pv[1, 64, 64] = nan, inf, inf
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    got = t.out.cpu()
    a, z = got[:, :, : hq // 2], got[:, :, hq // 2:]
    assert (a[..., 3] == inf).all() and (a[..., 9] == -inf).all() and torch.isnan(a[..., 20]).all()
    assert torch.isnan(z[..., 100]).all() and (z[..., 64] == inf).all()
    t.pv.nan_to_num_(0, 0, 0)
    out, lse, tol, tol_lse = t.want()
    rest = np.ones(got.shape, bool)
    rest[:, :, : hq // 2, [3, 9, 20]] = False
    rest[:, :, hq // 2:, [100, 64]] = False
    assert (np.abs(got.double().numpy() - out)[rest] <= tol[rest]).all()


@pytest.mark.parametrize("kind", KINDS, ids=["halves", "stream", "phases"])
def test_attend_tree_edges_in_every_kernel(fa, kind):
    """A hidden NaN node, a NaN that some rows read, an empty mask, and rows far apart in size, in each of the kernels."""
    hq, hkv, N, n, prefix = kind
    masks = _trees(7, N, n)
    masks[0][1] = 0
    masks = [[m & ~(1 << (n - 1)) for m in row] for row in masks]
    t = Tree(hq, hkv, 64, n, prefix, [40] + [3] * (N - 1), masks, seed=4)
    t.q[0] *= 30  # the scores of one branch rise far past the others'
    for b, length in enumerate(t.suffix):
        t.sk[b, :, length + n - 1] = float("nan")
        t.sv[b, :, length + n - 1] = float("inf")
    t.place()
    t.call(t.plan(fa))
    t.sk.nan_to_num_(0, 0, 0), t.sv.nan_to_num_(0, 0, 0)
    _close(t, t.want())


@pytest.mark.parametrize("d", [64, 128])
def test_attend_any_set_of_nodes(fa, d):
    """Masks that no tree gives: nothing, later nodes, not the node itself, bits past the nodes."""
    n = 12
    rng = np.random.default_rng(d)
    masks = [[int(rng.integers(0, 1 << 63)) for _ in range(n)] for _ in range(3)]
    masks[0][:4] = [0, 1 << 11, (1 << 64) - 1, 0xfffffffffffff000]
    t = Tree(6, 2, d, n, 0, [0, 3, 40], masks, seed=d)
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    want = t.want()
    assert np.isneginf(want[1][0, 0]).all() and np.isneginf(want[1][0, 3]).all()  # bits past the nodes count as none
    _close(t, want)


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_attend_what_no_bit_shows_has_no_influence(fa, value, paged):
    n, hidden = 10, 6
    masks = [[m & ~(1 << hidden) for m in row] for row in _trees(1, 3, n)]
    t = Tree(8, 2, 128, n, 90, [20, 0, 50], masks, paged, seed=1, junk=value)
    for b, length in enumerate(t.suffix):
        t.sk[b, :, length + hidden] = value
        t.sv[b, :, length + hidden] = value
    t.place()
    t.call(t.plan(fa))
    t.sk.nan_to_num_(0, 0, 0), t.sv.nan_to_num_(0, 0, 0)
    _close(t, t.want())


@pytest.mark.parametrize("d", [64, 128])
def test_attend_a_nan_value_reaches_the_rows_that_read_it(fa, d):
    n, bad = 11, 4
    masks = _trees(2, 3, n)
    t = Tree(8, 2, d, n, 77, [5, 30, 0], masks, seed=2)
    t.sv[1, 0, 30 + bad, 3] = float("nan")
    t.place()
    t.call(t.plan(fa))
    got = t.out.cpu()
    t.sv[1, 0, 30 + bad, 3] = 0
    out, _, tol, _ = t.want()
    reads = np.array([[b == 1 and masks[b][i] >> bad & 1 for i in range(n)] for b in range(3)], bool)
    assert reads.any() and not reads[1].all()
    hit = torch.isnan(got).all(-1).numpy()
    assert hit[:, :, :4][reads].all() and not hit[:, :, 4:].any() and not hit[:, :, :4][~reads].any()
    rest = ~hit
    assert (np.abs(got.double().numpy() - out)[rest] <= tol[rest]).all()


def test_attend_a_chain_is_the_prefill(fa):
    n = 12
    t = Tree(10, 2, 128, n, 700, [30, 4, 0, 90], [[(2 << i) - 1 for i in range(n)]] * 4, seed=9)
    t.place()
    t.call(t.plan(fa))
    p = fa.Plan.prefill_plan(t.hq, t.hkv, t.d, t.N, n, t.prefix, t.cap, t.cap)
    out = torch.empty_like(t.out)
    p.prefill(t.dq, *t.cache, t.lens, out)
    want = t.want()
    _close(t, want)
    assert (np.abs(out.double().cpu().numpy() - want[0]) <= want[2]).all()


def test_attend_repeats_and_graphs(fa):
    """The same bits every time, also from a captured graph replayed between eager calls on changed lengths and masks."""
    t = Tree(10, 2, 128, 16, 900, [30, 64, 0], _trees(4, 3, 16), seed=4)
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    first = t.out.clone(), t.lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t.call(plan)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.call(plan)
    other_masks = _i64(_trees(5, 3, 16))
    keep_masks, keep_lens = t.dmasks.clone(), t.lens.clone()
    for _ in range(3):
        t.dmasks.copy_(other_masks)
        t.lens.copy_(_i32([1, 2, 3]))
        t.call(plan)
        second = t.out.clone()
        t.out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(t.out.view(torch.int32), second.view(torch.int32))  # (one branch now reads rows that hold NaN)
        t.dmasks.copy_(keep_masks)
        t.lens.copy_(keep_lens)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t.out, first[0]) and torch.equal(t.lse, first[1])
        assert not torch.equal(second, first[0])


def test_attend_flags_what_the_device_holds(fa):
    t = Tree(8, 2, 64, 4, 20, [10, 50], _trees(1, 2, 4), seed=3)
    t.place()
    plan = t.plan(fa, max_len=30 + 4)  # 50 is clamped to 30
    t.call(plan)
    assert plan.device_error() == fa.ERR_SUFFIX_CLAMPED
    t = Tree(8, 2, 64, 4, 20, [10, 20], _trees(1, 2, 4), paged=True, seed=3)
    t.place()
    plan = t.plan(fa)
    t.cache[2][1, -1] = 10 ** 6  # the last page of the second row: positions past the nodes
    last = (20 + 4 - 1) // 16
    t.cache[2][1, 2 + last] = -5
    t.call(plan)
    torch.cuda.synchronize()
    assert plan.device_error() == fa.ERR_BAD_PAGE


@pytest.mark.parametrize("blocks", [1, 7, 1000])
def test_attend_any_grid(fa, blocks):
    t = Tree(8, 2, 128, 5, 700, [30, 200], _trees(6, 2, 5), seed=6)
    t.place()
    t.call(t.plan(fa, blocks=blocks))
    _close(t, t.want())


def test_attend_scale_and_more_than_64_branches(fa):
    t = Tree(2, 1, 64, 3, 40, [i % 7 for i in range(70)], _trees(8, 70, 3), seed=8, scale=0.3)
    t.place()
    t.call(t.plan(fa))
    _close(t, t.want())


def test_plans_take_their_own_calls_only(fa):
    t = Tree(8, 2, 64, 4, 20, [10, 20], _trees(1, 2, 4), seed=3)
    t.place()
    plan, prefill = t.plan(fa), fa.Plan.prefill_plan(8, 2, 64, 2, 4, 20, t.cap, t.cap)
    with pytest.raises(fa.FkaError, match="fka_tree_attend"):
        plan.prefill(t.dq, *t.cache, t.lens, t.out)
    with pytest.raises(fa.FkaError, match="not a tree plan"):
        prefill.tree_attend(t.dq, *t.cache, t.lens, t.dmasks, t.out)
    with pytest.raises(fa.FkaError, match="not a paged tree plan"):
        fa._check(fa.raw_call("fka_tree_attend_paged", plan.handle, *[None] * 9))
    with pytest.raises(fa.FkaError, match="instruction-prefill"):
        plan.decode(t.dq, *t.cache, t.lens, t.out)
    p = Tree(8, 2, 64, 4, 20, [10, 20], _trees(1, 2, 4), paged=True, seed=3)
    p.place()
    paged = p.plan(fa)
    with pytest.raises(fa.FkaError, match="fka_tree_attend_paged"):
        paged.prefill_paged(p.dq, *p.cache, p.lens, p.out)
    with pytest.raises(fa.FkaError, match="contiguous buffers"):
        fa._check(fa.raw_call("fka_tree_attend", paged.handle, *[None] * 10))
    # tensors of other sizes than the plan's
    for bad, name in ((dict(dq=t.dq[:1]), "q"), (dict(dmasks=t.dmasks[:, :3]), "masks"), (dict(lens=t.lens[:1]), "suffix_len"),
                      (dict(out=t.out[:1]), "out"), (dict(lse=t.lse[:1]), "out_lse"), (dict(cache=[c[:, :1] for c in t.cache]), "prefix_k")):
        was = {key: getattr(t, key) for key in bad}
        t.__dict__.update(bad)
        with pytest.raises(ValueError, match=name):
            t.call(plan)
        t.__dict__.update(was)
    t.dmasks = t.dmasks.int()
    with pytest.raises(ValueError, match="i64"):
        t.call(plan)


def test_attend_without_a_prefix_takes_none_for_it(fa):
    t = Tree(4, 2, 64, 5, 0, [3, 9], _trees(2, 2, 5), seed=2)
    t.place()
    t.cache[:2] = None, None
    t.call(t.plan(fa))
    _close(t, t.want())


def test_attend_on_another_stream_and_two_plans_at_once(fa):
    made = [Tree(8, 2, 128, 7, 600 + i, [30, 10], _trees(i, 2, 7), seed=i) for i in range(2)]
    plans, streams = [], [torch.cuda.Stream() for _ in made]
    for t in made:
        t.place()
        plans.append(t.plan(fa))
    torch.cuda.synchronize()
    for _ in range(5):
        for t, plan, stream in zip(made, plans, streams):
            with torch.cuda.stream(stream):
                t.call(plan)
    torch.cuda.synchronize()
    for t in made:
        _close(t, t.want())


# ------------------------------------------------------------------------------------------------- accept

def _accept(parents, masks, tokens, targets):
    """The accepted nodes of one tree, and the token behind the last."""
    n = len(parents)
    right = {0}
    for i in range(1, n):
        a = parents[i]
        if 0 <= a < i and tokens[i] == targets[a] and not any(parents[j] == a and tokens[j] == tokens[i] for j in range(1, i)):
            right.add(i)
    path = [i for i in range(n) if i == 0 or all(j in right for j in range(n) if (masks[i] | 1 << i) >> j & 1)]
    return path, targets[path[-1]]


def _accept_case(rng, N, n, likely, words=50):
    trees = [_parents(rng, n) for _ in range(N)]
    targets = rng.integers(0, words, (N, n))
    tokens = rng.integers(0, words, (N, n))
    for b in range(N):
        for i in range(1, n):
            if trees[b][i] >= 0 and rng.random() < likely:
                tokens[b, i] = targets[b, trees[b][i]]
    return trees, tokens, targets


@pytest.mark.parametrize("advance", [False, True])
@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("hkv,d,N,n,likely", [(2, 64, 5, 8, 0.5), (8, 128, 3, 16, 0.8), (1, 128, 4, 1, 0.5), (3, 64, 2, 64, 0.97),
                                              (20, 128, 2, 64, 1.0), (1, 64, 70, 5, 0.3)], ids=str)
def test_accept(fa, hkv, d, N, n, likely, paged, advance):
    rng = np.random.default_rng(n + N)
    trees, tokens, targets = _accept_case(rng, N, n, likely)
    masks = [_masks(t) for t in trees]
    lens = rng.integers(0, 60, N)
    cap = int(lens.max()) + n + 2
    prefix = rng.integers(0, 40, N)
    path, count, nxt = (torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((N, n), (N,), (N,)))
    dlens, err = _i32(lens), _i32([0])
    args = (_i32(trees), _i64(masks), _i32(tokens), _i32(targets))
    bits = lambda *s: torch.randint(-2**15, 2**15, s, dtype=torch.int16)  # noqa: E731  (NaN patterns among them)
    if paged:
        first, each = -(-prefix // 16), -(-cap // 16)
        width = int(first.max()) + each
        ids = rng.permutation(N * width + 3)[: N * width].reshape(N, width)
        k, v = bits(N * width + 3, hkv, 16, d), bits(N * width + 3, hkv, 16, d)
        row = lambda c, b, u: c[ids[b, first[b] + u // 16], :, u % 16]  # noqa: E731
    else:
        k, v = bits(N, hkv, cap, d), bits(N, hkv, cap, d)
        row = lambda c, b, u: c[b, :, u]  # noqa: E731
    dk, dv = (x.cuda().view(torch.bfloat16) for x in (k, v))
    if paged:
        fa.tree_accept_paged(*args, dk, dv, _i32(ids), _i32(prefix), dlens, path, count, nxt, max_len=cap, advance=advance, err=err)
    else:
        fa.tree_accept(*args, dk, dv, dlens, path, count, nxt, advance=advance, err=err)
    moved = 0
    for b in range(N):
        want, behind = _accept(trees[b], masks[b], tokens[b], targets[b])
        assert path[b].tolist() == want + [-1] * (n - len(want))
        assert int(count[b]) == len(want) and int(nxt[b]) == behind
        assert int(dlens[b]) == lens[b] + (len(want) if advance else 0)
        for j, i in enumerate(want):
            for c in (k, v):
                row(c, b, int(lens[b]) + j)[...] = row(c, b, int(lens[b]) + i).clone()
            moved += i != j
    assert n == 1 or moved or likely < 0.4
    assert torch.equal(dk.view(torch.int16).cpu(), k) and torch.equal(dv.view(torch.int16).cpu(), v)
    assert int(err) == 0


def test_accept_takes_the_first_of_two_equal_children_and_no_child_of_an_unused_node(fa):
    parents = [[-1, 0, 0, 1, 2, -1, 5, 3, 3], [-1, -1, 0, 0, 2, 3, -1, 6, 5]]
    tokens = [[0, 7, 7, 8, 8, 7, 1, 9, 9], [0, 4, 4, 5, 1, 2, 9, 9, 3]]
    targets = [[7, 8, 8, 9, 1, 1, 1, 6, 6], [5, 1, 1, 2, 1, 3, 9, 1, 77]]
    masks = [_masks(p) for p in parents]
    k = torch.zeros(2, 1, 20, 64, dtype=torch.bfloat16, device="cuda")
    path, count, nxt, lens = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, 9), (2,), (2,), (2,)))
    fa.tree_accept(_i32(parents), _i64(masks), _i32(tokens), _i32(targets), k, k.clone(), lens, path, count, nxt)
    assert path.tolist() == [[0, 1, 3, 7] + [-1] * 5, [0, 3, 5, 8] + [-1] * 5]
    assert nxt.tolist() == [6, 77] and lens.tolist() == [4, 4]


def test_accept_without_room_or_pages(fa):
    n, N = 4, 4
    trees, tokens, targets = [[-1, 0, 1, 2]] * N, [[5, 6, 7, 8]] * N, [[6, 7, 8, 9]] * N
    args = (_i32(trees), _i64([_masks(t) for t in trees]), _i32(tokens), _i32(targets))
    new = lambda: tuple(torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((N, n), (N,), (N,)))  # noqa: E731
    k = torch.arange(N * 20 * 64, device="cuda").view(N, 1, 20, 64).bfloat16()
    v, before = k.clone(), k.clone()
    path, count, nxt = new()
    lens, err = _i32([16, 17, -1, 2**31 - 1]), _i32([0])
    fa.tree_accept(*args, k, v, lens, path, count, nxt, err=err)
    assert count.tolist() == [4, 0, 0, 0] and nxt.tolist() == [9, -1, -1, -1] and path[1:].eq(-1).all()
    assert lens.tolist() == [20, 17, -1, 2**31 - 1] and int(err) == fa.ERR_APPEND_NO_ROOM and torch.equal(k, before)
    # pages: one past the pool, one negative, one past the table
    pool = torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    path, count, nxt = new()
    lens, err = _i32([14, 14, 14, 30]), _i32([0])
    table = _i32([[0, 1], [0, 4], [-1, 2], [2, 3]])
    fa.tree_accept_paged(*args, pool, pool.clone(), table, _i32([0] * N), lens, path, count, nxt, max_len=1000, err=err)
    assert count.tolist() == [4, 0, 0, 0] and lens.tolist() == [18, 14, 14, 30] and int(err) == fa.ERR_APPEND_NO_ROOM


def test_accept_from_a_graph(fa):
    rng = np.random.default_rng(1)
    trees, tokens, targets = _accept_case(rng, 3, 16, 0.9)
    args = (_i32(trees), _i64([_masks(t) for t in trees]), _i32(tokens), _i32(targets))
    k = torch.randn(3, 2, 100, 128, device="cuda").bfloat16()
    v, lens = k.clone(), _i32([0, 7, 20])
    path, count, nxt = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((3, 16), (3,), (3,)))
    state = (k, v, lens)
    start = [x.clone() for x in state]
    fa.tree_accept(*args, k, v, lens, path, count, nxt)
    want = [x.clone() for x in state + (path, count, nxt)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fa.tree_accept(*args, k, v, lens, path, count, nxt)
    for _ in range(3):
        for x, y in zip(state, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(state + (path, count, nxt), want))


def test_accept_past_four_gib(fa):
    """Rows behind 2^32 bytes of a cache."""
    n, hkv, d, cap = 6, 4, 128, 2_200_000
    k = torch.empty(2, hkv, cap, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    lens = [cap - 10, cap - n]
    parents, tokens, targets = [[-1, 0, 0, 2, 3, 4]] * 2, [[9, 1, 2, 3, 4, 5]] * 2, [[2, 0, 3, 4, 5, 6]] * 2
    want = []
    for b, length in enumerate(lens):
        for c in (k, v):
            c[b, :, length: length + n] = torch.randn(hkv, n, d, device="cuda")
            want.append(c[b, :, [length + i for i in (0, 2, 3, 4, 5)]].clone())
    dlens, (path, count, nxt) = _i32(lens), (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((2, n), (2,), (2,)))
    fa.tree_accept(_i32(parents), _i64([_masks(p) for p in parents]), _i32(tokens), _i32(targets), k, v, dlens, path, count, nxt)
    assert count.tolist() == [5, 5] and nxt.tolist() == [6, 6]
    got = [c[b, :, length: length + 5] for b, length in enumerate(lens) for c in (k, v)]
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("hq,n", [(4, 3), (32, 20)], ids=["halves", "phases"])
def test_attend_past_four_gib(fa, hq, n, paged):
    """The keys that count are behind 2^32 bytes of a prefix; those in front have less than 2^-90 of their weight."""
    near, L = 300, 4_200_003
    t = Tree(hq, 4, 128, n, near, [5], _trees(3, 1, n), scale=1.0, junk=0.0)
    t.q[..., 0] = 8
    t.pk[..., 0] = t.sk[..., 0] = 0
    t.place()
    if paged:
        shared = -(-L // 16)
        cache = []
        for pre, suf in ((t.cache[0], t.cache[2]), (t.cache[1], t.cache[3])):
            pool = torch.zeros(shared + 3, 4, 16, 128, dtype=torch.bfloat16, device="cuda")
            if not cache:
                pool[:shared, :, :, 0] = -8
            for i in range(near):
                at = L - near + i
                pool[at // 16, :, at % 16] = pre[:, i]
            for u in range(t.cap):
                pool[shared + 2 - u // 16, :, u % 16] = suf[0, :, u]
            cache.append(pool)
        pages = -(-t.cap // 16)
        table = torch.cat([torch.arange(shared), shared + 2 - torch.arange(pages)]).to(torch.int32).cuda()[None].contiguous()
        plan = fa.Plan.tree_paged_plan(hq, 4, 128, 1, n, L, table.shape[1], shared + 3, t.cap, softmax_scale=1.0)
        plan.tree_attend_paged(t.dq, *cache, table, t.lens, t.dmasks, t.out, t.lse)
    else:
        k, v = (torch.zeros(4, L, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        k[..., 0] = -8
        k[:, L - near:], v[:, L - near:] = t.cache[0], t.cache[1]
        plan = fa.Plan.tree_plan(hq, 4, 128, 1, n, L, t.cap, t.cap, softmax_scale=1.0)
        plan.tree_attend(t.dq, k, v, t.cache[2], t.cache[3], t.lens, t.dmasks, t.out, t.lse)
    _close(t, t.want())


def _bf16_round(x):
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def _adverse_keys():
    """64 scores whose p = exp(score) lose the most in two bf16 terms (62 of them, and 0 at places 0 and 32, each half's largest), and
    values of 1 and -1 with the sign of what is lost: the losses add up, while the sums of p v stay near 0."""
    bits = np.arange(0xbc01, 0xbf30, dtype=np.uint32) << 16  # bf16 from -0.69 to -2^-7
    x = bits.view(np.float32).astype(np.float64)
    x = x[(x > -0.69) & (x < -2.0 ** -7)]
    p = np.exp(x)
    hi = _bf16_round(p)
    lost = p - hi - _bf16_round(p - hi)
    picks = [sorted(np.nonzero(lost * sign > 0)[0][np.argsort(-lost[lost * sign > 0] * sign)][:31], key=lambda i: p[i]) for sign in (1, -1)]
    pairs = [i for both in zip(*picks) for i in both]
    s = np.concatenate([[0], x[pairs[:31]], [0], x[pairs[31:]]])
    v = np.concatenate([[1], np.sign(lost[pairs[:31]]), [-1], np.sign(lost[pairs[31:]])])
    return s, v, np.abs(lost[pairs]).sum() / np.exp(s).sum()


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,N", [(4, 2, 2), (64, 1, 3)], ids=["halves", "stream"])
def test_attend_of_few_rows_keeps_three_terms_of_p(fa, hq, hkv, N, d, paged):
    """A score is one exact product, 64 keys a row.  What a result is off by, in parts of the sum of p (55): p's exponential (a last bit, 2^-23), its argument in (-1, 0]
    and the scale (2^-25 each, times ln 2) and the third term (2^-27) come to 1.8e-7; six products over 32 keys add in at most 192 roundings of partial sums
    of at most 3.2, the signs alternating, 6.7e-7.  The division, and a merge of two halves, scale a result near 0.  2^-20 holds all of that; two
    terms lose four times as much."""
    s, v, lost = _adverse_keys()
    assert np.abs(np.cumsum(np.exp(s) * v)).max() < 3.2 and lost > 4 * 2.0 ** -20
    t = Tree(hq, hkv, d, 1, 0, [63] * N, [[1]] * N, paged, scale=1.0)
    t.q.zero_()
    t.q[..., 0] = 1
    t.sk[:, :, :64, 0] = torch.from_numpy(s).bfloat16()
    t.sv[:, :, :64] = torch.from_numpy(v).bfloat16()[:, None]
    assert torch.equal(t.sk[0, 0, :64, 0].double(), torch.from_numpy(s))
    t.place()
    t.call(t.plan(fa))
    want = float((np.exp(s) * v).sum() / np.exp(s).sum())
    assert float((t.out.double() - want).abs().max()) <= 2.0 ** -20


def test_plans_keep_their_partial_results_below_256_mib(fa):
    """However many blocks the caller asks for, also where two waves share a unit and write a part each."""
    for heads, n, paged in (((128, 64, 128), 64, False), ((128, 64, 128), 64, True), ((64, 64, 64), 8, False), ((640, 64, 128), 16, False)):
        if paged:
            plan = fa.Plan.tree_paged_plan(*heads, 1, n, 64 * 300, 1300, 1300, n, blocks=64 * 300)
        else:
            plan = fa.Plan.tree_plan(*heads, 1, n, 64 * 300, n, n, blocks=64 * 300)
        info = plan.info()
        rows = n * heads[0] * info.n_slots
        assert info.n_slots > 8 and rows * heads[2] * 4 <= 256 << 20 and info.workspace_bytes <= (256 << 20) + rows * 4 + (8 << 20)
        plan.close()


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
def test_attend_refuses_outputs_upon_what_outlives_the_call(fa, paged):
    """out and out_lse upon each other, the caches, the page table, the lengths and the masks; behind or upon q they may be."""
    t = Tree(8, 2, 64, 4, 64, [10, 20], _trees(1, 2, 4), paged, seed=3)
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    torch.cuda.synchronize()
    want, lse = t.out.clone(), t.lse.clone()
    inputs = dict(zip(("k_pool", "v_pool", "page_table") if paged else ("prefix_k", "prefix_v", "suffix_k", "suffix_v"), t.cache),
                  suffix_len=t.lens, masks=t.dmasks)
    name = "fka_tree_attend_paged" if paged else "fka_tree_attend"
    tail = [t.lens.data_ptr(), t.dmasks.data_ptr()]

    def call(out, out_lse):
        return fa.raw_call(name, plan.handle, t.dq.data_ptr(), *[c.data_ptr() for c in t.cache], *tail, out, out_lse, None)

    for what, x in inputs.items():
        size = x.numel() * x.element_size()
        for at in (x.data_ptr(), x.data_ptr() + (size - 1) // 16 * 16):
            assert call(at, t.lse.data_ptr()) == -1 and f"out overlaps {what}" in fa.last_error()
            assert call(t.out.data_ptr(), at) == -1 and f"out_lse overlaps {what}" in fa.last_error()
    assert call(t.out.data_ptr(), t.out.data_ptr() + 4 * t.out.numel() - 4) == -1 and "out overlaps out_lse" in fa.last_error()
    # q at the start of out's memory
    both = torch.empty_like(t.out)
    t.dq = both.view(-1).view(torch.bfloat16)[: t.q.numel()].view(t.q.shape)
    t.dq.copy_(t.q)
    t.out = both
    t.call(plan)
    assert torch.equal(t.out, want) and torch.equal(t.lse, lse)


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", KINDS, ids=["halves", "stream", "phases"])
def test_attend_infinite_suffix_values(fa, kind, d, paged):
    """An infinity of a suffix or node's V is that infinity in its channel of the rows that read its key, both signs there are NaN, and nothing else changes."""
    hq, hkv, N, n, prefix = kind
    masks = _trees(11, N, n)
    t = Tree(hq, hkv, d, n, prefix, [70, 5, 0, 33, 12][:N], masks, paged, seed=3)
    inf = float("inf")
    plants = [  # branch (None: the prefix), suffix position, KV head, channel, value
        (0, 2, 0, 3, inf), (0, 69, 0, d - 1, -inf), (0, 64, 0, 17, inf), (0, 1, 0, 17, -inf),  # committed, the last of them of both signs
        (1, 5 + n - 1, 1, 9, -inf), (1, 5, 1, 20, inf),                                        # the last node, the root
        (2, 1, 0, 30, inf), (2, 0, 0, 30, -inf), (2, 2, 1, 31, -inf),                          # nodes of both signs, no committed key
        (None, 100, 1, 40, inf), (0, 7, 1, 40, -inf), (1, 3, 1, 40, inf),                      # one in the prefix too
    ]
    for b, u, g, c, x in plants:
        (t.pv[g] if b is None else t.sv[b, g])[u, c] = x
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    for b, u, g, c, _ in plants:
        (t.pv[g] if b is None else t.sv[b, g])[u, c] = 0
    out, lse, tol, tol_lse = t.want()
    G = hq // hkv
    for row in np.ndindex(N, n):
        for b, u, g, c, x in plants:
            at = u - t.suffix[row[0]]
            if b is None or b == row[0] and (at < 0 or int(masks[b][row[1]]) >> at & 1):
                with np.errstate(invalid="ignore"):
                    out[row][g * G: (g + 1) * G, c] += x
    special = ~np.isfinite(out)
    got = t.out.double().cpu().numpy()
    assert special.any(-1).any(-1).sum() >= N and np.isnan(out).any() and np.isinf(out).any()
    assert np.array_equal(got[special], out[special], equal_nan=True)
    assert (np.abs(got[~special] - out[~special]) <= tol[~special]).all()
    assert (np.abs(t.lse.double().cpu().numpy() - lse) <= tol_lse).all()
    assert plan.device_error() == 0


@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
@pytest.mark.parametrize("N,n", [(200, 1), (100, 2)])
def test_attend_more_than_64_branches_in_one_block(fa, N, n, paged):
    """One query row to a token: a block's rows are of 200 or 100 branches, more than a wave has lanes."""
    t = Tree(2, 2, 64, n, 40, [i % 7 for i in range(N)], _trees(8, N, n), paged, seed=n)
    bad = 94  # (suffix of 3)
    t.sv[bad, 1, 1, 5] = float("inf")
    t.place()
    plan = t.plan(fa)
    t.call(plan)
    assert (t.out[bad, :, 1, 5] == float("inf")).all()
    t.sv[bad, 1, 1, 5] = 0
    want = t.want()
    t.out[bad, :, 1, 5] = torch.from_numpy(want[0][bad, :, 1, 5]).float().cuda()
    _close(t, want)
    assert plan.device_error() == 0
