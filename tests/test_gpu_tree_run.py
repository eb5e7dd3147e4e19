"""The operators of drafted trees together, as a serving program runs them: a small model of one attention layer decodes greedily,
token by token with the plain step, and again with trees of drafted tokens, some of them right.  Both give the same tokens,
and after each step the same cache rows bit for bit."""
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HQ, HKV, D, WORDS, PREFIX, N = 8, 2, 64, 300, 150, 3


@pytest.fixture(scope="module")
def fa():
    from paper_2608_13667_amd import forkattn
    return forkattn


class Model:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.embed = r(WORDS, (HQ + 2 * HKV) * D).bfloat16().cuda()  # a token's q, k and v
        self.out = r(HQ * D, WORDS).cuda()
        self.freq = (1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).cuda()
        self.prefix_k, self.prefix_v = r(HKV, PREFIX, D).bfloat16().cuda(), r(HKV, PREFIX, D).bfloat16().cuda()

    def project(self, tokens):
        rows = self.embed[tokens.long()]
        heads = lambda a, z, n: rows[..., a * D: z * D].unflatten(-1, (n, D))  # noqa: E731
        return heads(0, HQ, HQ), heads(HQ, HQ + HKV, HKV), heads(HQ + HKV, HQ + 2 * HKV, HKV)

    def logits(self, o):
        return o.flatten(-2) @ self.out


class Cache:
    """Suffixes in buffers, or behind the prefix in the pages of a pool."""

    def __init__(self, m, cap, paged, seed):
        self.cap, self.paged = cap, paged
        self.lens = torch.zeros(N, dtype=torch.int32, device="cuda")
        if not paged:
            self.k, self.v = (torch.zeros(N, HKV, cap, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
            return
        shared, each = -(-PREFIX // 16), -(-cap // 16)
        ids = np.random.default_rng(seed).permutation(shared + N * each)
        self.k, self.v = (torch.zeros(len(ids), HKV, 16, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        for p in range(PREFIX):
            self.k[ids[p // 16], :, p % 16], self.v[ids[p // 16], :, p % 16] = m.prefix_k[:, p], m.prefix_v[:, p]
        rows = [np.concatenate([ids[:shared], ids[shared + b * each: shared + (b + 1) * each]]) for b in range(N)]
        self.table = torch.tensor(np.array(rows, np.int32), device="cuda")
        self.prefix_len = torch.full((N,), PREFIX, dtype=torch.int32, device="cuda")
        self.shared = shared

    def rows(self):
        """Each branch's committed rows of K and V."""
        got = []
        for b, n in enumerate(self.lens.tolist()):
            for c in (self.k, self.v):
                if self.paged:
                    c = c[self.table[b, self.shared:].long()].transpose(0, 1).flatten(1, 2)
                    got.append(c[:, :n].clone())
                else:
                    got.append(c[b, :, :n].clone())
        return got

    def store(self, fa, q, k, v, positions, freq):
        q_out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        if self.paged:
            fa.rotate_append_paged(q, k, v, positions, freq, q_out, self.k, self.v, self.table, self.prefix_len, self.lens)
        else:
            fa.rotate_append(q, k, v, positions, freq, q_out, self.k, self.v, self.lens)
        return q_out


def _greedy(fa, logits, work):
    tokens = torch.empty(logits.shape[0], dtype=torch.int32, device="cuda")
    fa.sample(logits, torch.zeros(logits.shape[0], device="cuda"), tokens, workspace=work,
              temperature=torch.zeros(logits.shape[0], device="cuda"))
    return tokens


def _one_by_one(fa, m, first, steps):
    """The tokens that follow `first`, and the cache rows of all of them but the last."""
    cache = Cache(m, steps + 1, False, 0)
    plan = fa.Plan.contig(HQ, HKV, D, N, PREFIX, cache.cap, cache.cap)
    out, work = torch.empty(N, HQ, D, device="cuda"), fa.sample_workspace(N, WORDS)
    token, said = first, [first.clone()]
    for _ in range(steps):
        q, k, v = m.project(token[:, None])
        q = cache.store(fa, q, k, v, (PREFIX + cache.lens)[:, None].contiguous(), m.freq)
        cache.lens += 1
        plan.decode(q[:, 0].contiguous(), m.prefix_k, m.prefix_v, cache.k, cache.v, cache.lens, out)
        token = _greedy(fa, m.logits(out), work)
        said.append(token.clone())
    return torch.stack(said, 1), cache


@pytest.mark.parametrize("n", [1, 7, 24])
@pytest.mark.parametrize("paged", [False, True], ids=["contiguous", "paged"])
def test_trees_decode_what_single_tokens_do(fa, paged, n):
    m, steps = Model(3), 30
    first = torch.tensor([5, 17, 200], dtype=torch.int32, device="cuda")
    said, single = _one_by_one(fa, m, first, steps + n)
    truth, want = said.tolist(), single.rows()
    rng = np.random.default_rng(n)
    cache = Cache(m, steps + 2 * n + 2, paged, 1)
    make = (HQ, HKV, D, N, n, PREFIX)
    plan = fa.Plan.tree_paged_plan(*make, cache.table.shape[1], cache.k.shape[0], cache.cap) if paged else \
        fa.Plan.tree_plan(*make, cache.cap, cache.cap)
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
    masks, positions, path, count, pending = torch.empty(N, n, dtype=torch.int64, device="cuda"), i32(N, n), i32(N, n), i32(N), first.clone()
    out, work, err = torch.empty(N, n, HQ, D, device="cuda"), fa.sample_workspace(N * n, WORDS), torch.zeros(1, dtype=torch.int32, device="cuda")
    got, accepted = [[] for _ in range(N)], 0
    for _ in range(steps):
        done = [len(g) for g in got]
        if max(done) >= steps:
            break
        # drafts: behind each node wrong words and, mostly, the right one
        parents, tokens = np.full((N, n), -1, np.int32), np.zeros((N, n), np.int32)
        for b in range(N):
            tokens[b, 0] = int(pending[b])
            depth, right = {0: 0}, {0}
            for i in range(1, n):
                if rng.random() < 0.1:
                    tokens[b, i] = rng.integers(WORDS)  # a place that is not used
                    continue
                a = int(rng.choice(sorted(depth)[-4:]))
                parents[b, i], depth[i] = a, depth[a] + 1
                true = truth[b][done[b] + depth[i]]
                tokens[b, i] = true if rng.random() < 0.6 else rng.integers(WORDS)
                if a in right and tokens[b, i] == true:
                    right.add(i)
        dp, dt = torch.tensor(parents, device="cuda"), torch.tensor(tokens, device="cuda")
        fa.tree_layout(dp, PREFIX + cache.lens, masks, positions, err=err)
        q = cache.store(fa, *m.project(dt), positions, m.freq)
        if paged:
            plan.tree_attend_paged(q, cache.k, cache.v, cache.table, cache.lens, masks, out)
            fa_accept, where = fa.tree_accept_paged, (cache.k, cache.v, cache.table, cache.prefix_len)
        else:
            plan.tree_attend(q, m.prefix_k, m.prefix_v, cache.k, cache.v, cache.lens, masks, out)
            fa_accept, where = fa.tree_accept, (cache.k, cache.v)
        targets = _greedy(fa, m.logits(out.view(N * n, HQ, D)), work).view(N, n)
        fa_accept(dp, masks, dt, targets, *where, cache.lens, path, count, pending, err=err)
        for b in range(N):
            nodes = [i for i in path[b].tolist() if i >= 0]
            assert len(nodes) == int(count[b]) >= 1 and nodes[0] == 0
            got[b] += [int(tokens[b, i]) for i in nodes]
            accepted += len(nodes) - 1
        # the committed tokens and the pending one are those of the single steps, and so are the cache's rows
        for b in range(N):
            assert got[b] + [int(pending[b])] == truth[b][: len(got[b]) + 1]
        for have, all_rows in zip(cache.rows(), want):
            assert torch.equal(have, all_rows[:, : have.shape[1]])
    assert cache.lens.tolist() == [len(g) for g in got]
    assert accepted > 0 or n == 1
    assert int(err) == 0 and plan.device_error() == 0


class Layer:
    """One of several layers that share the lengths; `rest` keeps what the cache holds when the nodes are in it."""

    def __init__(self, g, heads, d, n_branches, n, prefix_len, cap):
        hq, hkv = heads
        r = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
        self.new = r(n_branches, n, hq, d), r(n_branches, n, hkv, d), r(n_branches, n, hkv, d)
        self.prefix_k, self.prefix_v = r(hkv, prefix_len, d), r(hkv, prefix_len, d)
        self.suffix_k, self.suffix_v = r(n_branches, hkv, cap, d), r(n_branches, hkv, cap, d)

    def project(self, hidden):
        return self.new

    def rest(self, hidden, out):
        self.before = self.suffix_k.clone(), self.suffix_v.clone()
        return hidden


def test_the_documented_step_through_several_layers(fa):
    """The step of README.md as it stands there, three layers: each layer's accepted rows move together, the lengths advance once."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    step = text[text.index("A step with drafted trees"):].split("```python\n")[1].split("```")[0]
    n_q_heads, n_kv_heads, d, n_branches, n, prefix_len, cap, max_len, vocab = 8, 2, 64, 3, 9, 100, 64, 64, WORDS
    g = torch.Generator().manual_seed(1)
    layers = [Layer(g, (n_q_heads, n_kv_heads), d, n_branches, n, prefix_len, cap) for _ in range(3)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    start = [0, 17, 40]
    logits = torch.full((n_branches * n, vocab), -5.0, device="cuda")
    said = torch.randint(vocab, (n_branches, n), generator=g)  # behind each node
    logits[torch.arange(n_branches * n, device="cuda"), said.flatten().cuda()] = 9.0
    parents = [[-1, 0, 0, 2, 3, 2, 5, 4, 7]] * n_branches
    tokens = said.new_zeros(n_branches, n)
    for b in range(n_branches):
        for i in range(1, n):  # wrong at the first child, and (branch by branch) from some depth on
            tokens[b, i] = (said[b, parents[b][i]] + (i == 1 or i in (5, 6) or (b == 1 and i >= 7))) % vocab
    names = dict(fa=fa, torch=torch, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, d=d, n_branches=n_branches, n=n, prefix_len=prefix_len, cap=cap,
                 max_len=max_len, vocab=vocab, layers=layers, hidden=None, head=lambda hidden: logits, parents=i32(parents), base=i32(start) + prefix_len,
                 tokens=i32(tokens.tolist()), suffix_len=i32(start), u=torch.zeros(n_branches * n, device="cuda"),
                 t=torch.zeros(n_branches * n, device="cuda"), p=torch.ones(n_branches * n, device="cuda"),
                 freq=(1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).cuda(),
                 masks=torch.empty(n_branches, n, dtype=torch.int64, device="cuda"), q_rot=torch.empty(n_branches, n, n_q_heads, d, dtype=torch.bfloat16, device="cuda"),
                 out=torch.empty(n_branches, n, n_q_heads, d, device="cuda"))
    for name in ("positions", "path"):
        names[name] = torch.empty(n_branches, n, dtype=torch.int32, device="cuda")
    names.update(targets=torch.empty(n_branches * n, dtype=torch.int32, device="cuda"), count=i32([0] * n_branches), next_token=i32([0] * n_branches))
    exec(step, names)
    want = [[0, 2, 3, 4, 7, 8], [0, 2, 3, 4], [0, 2, 3, 4, 7, 8]]
    assert names["path"].tolist() == [w + [-1] * (n - len(w)) for w in want] and names["count"].tolist() == [len(w) for w in want]
    assert names["suffix_len"].tolist() == [s + len(w) for s, w in zip(start, want)]
    assert names["next_token"].tolist() == [int(said[b, w[-1]]) for b, w in enumerate(want)]
    for layer in layers:
        for cache, before in zip((layer.suffix_k, layer.suffix_v), layer.before):
            for b, (s, w) in enumerate(zip(start, want)):
                before[b, :, s: s + len(w)] = before[b, :, [s + i for i in w]].clone()
            assert torch.equal(cache, before)
