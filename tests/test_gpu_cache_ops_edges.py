"""Edges of the operators around a snapshot's cache on the GPU: values, magnitudes and sizes at which a result is easily lost.
Tolerances as in tests/test_gpu_cache_ops.py, or derived beside the test."""
import numpy as np
import pytest
import torch

from tests.gpu_util import dev_bf16, dev_i32
from tests.test_gpu_cache_ops import (Mx, bits_of, close_rotated, fa, host, normal, ref_evict,  # noqa: F401  (fa is the fixture)
                                      ref_rotate, value)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hkv,G,N", [(64, 2, 5, 5), (128, 2, 5, 5), (128, 2, 20, 3), (128, 1, 12, 5), (64, 1, 64, 1)])
@pytest.mark.parametrize("step", [False, True])
def test_mx_infinite_suffix_values(fa, step, d, hkv, G, N):  # noqa: F811
    """An infinite value in a suffix is its channel's result in the rows that read it, as the sum says; infinities of both signs give NaN;
    nothing else changes."""
    rng = np.random.default_rng(80 + G)
    lens = [5, 90, 700, 0, 33][-N:]
    m = Mx(fa, 81 + G, G * hkv, hkv, d, [N], [300], lens, cap=720)
    s = int(np.argmax(lens))  # the sequence, over several blocks where they share it
    kn, vn = normal(rng, N, hkv, d), normal(rng, N, hkv, d)
    lens0 = m.dev["suffix_len"].clone()

    def run():
        out, lse = m.outs()
        m.dev["suffix_len"].copy_(lens0)
        if step:
            m.plan.step_mx(m.dev["q"], dev_bf16(kn), dev_bf16(vn), m.tiles, m.dev["suffix_k"], m.dev["suffix_v"],
                           m.dev["suffix_len"], out, lse)
        else:
            m.plan.decode_mx(out=out, out_lse=lse, **m.dev)
        return out.cpu().numpy(), lse.cpu().numpy()

    want, want_lse = run()
    inf, last, g = float("inf"), int(lens[s]) - 1, hkv - 1
    rows = np.s_[s, g * G: (g + 1) * G]
    for c, places in ((7, {5: inf}), (d - 1, {3: -inf}), (20, {0: inf, last: inf, 11: inf}), (33, {last: -inf}), (11, {4: inf, last: -inf}),
                      (12, {6: inf, 7: -inf})):
        for k, x in places.items():
            m.dev["suffix_v"][s, g, k, c] = x
        signs = set(places.values())
        want[rows + (c,)] = signs.pop() if len(signs) == 1 else np.nan
    if step:  # the new token's
        vn[s, g, 1], vn[s, g, 7] = 0x7F80, 0xFF80
        want[rows + (1,)], want[rows + (7,)] = inf, np.nan
    out, lse = run()
    assert np.array_equal(out, want, equal_nan=True), np.argwhere((out != want) & ~(np.isnan(out) & np.isnan(want)))[:8]
    assert np.array_equal(lse, want_lse)


@pytest.mark.parametrize("d", [64, 128])
def test_mx_small_weights_add_up(fa, d):  # noqa: F811
    """One key with 2^16 times the weight of any other and half a million of those beside it, all values 1: the output is 1.  A wave sums half of them
    in n / 64 steps of products, and a lane n / 64 numbers: roundings of either sign, each at most half a step of the sum (2^-24, a standard
    deviation of 2^-23 / sqrt(12)), in all sqrt(n / 32) of that in a row; what loses a part of each small weight shows in the mean
    over the rows, which is held to six deviations of its own."""
    n, hkv, G, N = 1 << 19, 2, 16, 4
    gen = torch.Generator(device="cuda")
    gen.manual_seed(90 + d)
    k = torch.zeros(hkv, n, d, dtype=torch.bfloat16, device="cuda")
    k[..., 32:64].normal_(generator=gen)
    k[:, 0, 32:64], k[:, 0, 0] = 0, 6
    q = torch.zeros(N, hkv * G, d, dtype=torch.bfloat16, device="cuda")
    q[..., 32:64].normal_(std=0.1, generator=gen)
    q[..., 0] = 11 / 6  # the others have some 2^-16 of that key's weight each, 10 times as much together
    tiles = torch.empty(n // 128, hkv, 136 * d, dtype=torch.uint8, device="cuda")
    fa.mx_pack(k, torch.ones_like(k), tiles)
    plan = fa.Plan.mx_plan(hkv * G, hkv, d, [0, N], [n], 1, 0, n_pool_tiles=n // 128, softmax_scale=1.0, blocks=1)
    suffix = torch.zeros(N, hkv, 1, d, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty(N, hkv * G, d, device="cuda"), torch.empty(N, hkv * G, device="cuda")
    plan.decode_mx(q, tiles, suffix, suffix, dev_i32([0] * N), out, lse)
    err = out.cpu().numpy().astype(np.float64)[..., 0] - 1
    dev = np.sqrt(n / 32) * 2.0 ** -23 / np.sqrt(12)
    print(f"[small weights] mean {err.mean():.2e} of {6 * dev / np.sqrt(err.size):.2e}, worst {np.abs(err).max():.2e} of {6 * dev:.2e}", flush=True)
    assert abs(err.mean()) <= 6 * dev / np.sqrt(err.size) and np.abs(err).max() <= 6 * dev
    assert (out == out[..., :1]).all()


@pytest.mark.parametrize("where", ["prefix", "suffix", "wide prefix"])
@pytest.mark.parametrize("d", [64, 128])
def test_mx_products_keep_all_of_p(fa, d, where):  # noqa: F811
    """Three keys whose scores are exact in fp32 and close to each other, values 1 and -1: what is left is the error of p and of its terms.
    A weight: its exponent, below 8, is off by 2^-22 (half a step) and by 2^-24 of at most 1 (the scale), times ln 2, the exponential by
    2^-23; its terms by 2^-23 at most; then 16 fp32 steps of sums, reciprocals and joins.  A term of p less is off by 2^-18 of p
    (suffixes, values outside fp16's range: three bf16 terms) or by 2^-12 (two fp16 terms), and fails."""
    rng = np.random.default_rng(95)
    hkv, G, N, n, scale = 8, 8, 8, 3, 2.0 ** -6
    grid = lambda step, top, *s: np.clip(np.round(rng.standard_normal(s) / step) * step, -top, top)  # noqa: E731
    # the values of a block come back as they are: 0, 0.5, .. 6 under one scale
    size = 2.0 ** 40 if where == "wide prefix" else 1.0
    v = np.where(rng.random((hkv, n, d)) < 0.5, -size, size)
    q, k = grid(0.25, 2, N, hkv * G, d), grid(0.5, 2, hkv, n, d)
    to_bits = lambda x: torch.from_numpy(np.asarray(x, np.float32)).bfloat16().cuda()  # noqa: E731
    prefix = 0 if where == "suffix" else n
    plan = fa.Plan.mx_plan(hkv * G, hkv, d, [0, N], [prefix], n, n, n_pool_tiles=1, softmax_scale=scale)
    tiles = torch.zeros(1, hkv, 136 * d, dtype=torch.uint8, device="cuda")
    sk, sv = torch.zeros(N, hkv, n, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(N, hkv, n, d, dtype=torch.bfloat16, device="cuda")
    if prefix:
        fa.mx_pack(to_bits(k), to_bits(v), tiles)
        back = [torch.empty(hkv, n, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        fa.mx_unpack(tiles, *back)
        assert torch.equal(back[0], to_bits(k)) and torch.equal(back[1], to_bits(v))
    else:
        sk[:], sv[:] = to_bits(k), to_bits(v)
    out, lse = torch.empty(N, hkv * G, d, device="cuda"), torch.empty(N, hkv * G, device="cuda")
    plan.decode_mx(to_bits(q), tiles, sk, sv, dev_i32([0 if prefix else n] * N), out, lse)
    w = np.exp(scale * np.matmul(q.reshape(N, hkv, G, d), k.transpose(0, 2, 1)[None]))
    total = w.sum(-1, keepdims=True)
    ref = np.matmul(w / total, v[None]).reshape(N, hkv * G, d)
    tol = ((2.0 ** -22 + 2.0 ** -24) * np.log(2) + 2.0 ** -23 + 2.0 ** -23 + 16 * 2.0 ** -24) * size
    err = np.abs(out.cpu().numpy() - ref).max()
    print(f"[terms of p] d {d} {where}: {err / size:.2e} of {tol / size:.2e}", flush=True)
    assert err <= tol
    assert np.abs(lse.cpu().numpy().reshape(N, hkv, G) - np.log(total)[..., 0]).max() <= 2.0 ** -19


def test_mx_pool_without_room_for_the_prefixes(fa):  # noqa: F811
    """Without a tile table the ids are known: a pool with fewer tiles is refused, by the decode and the step, and nothing runs; with a
    table the same plan works."""
    m = Mx(fa, 97, 8, 2, 64, [2, 1], [300, 129], [3, 4, 5])  # 3 + 2 tiles
    kn = dev_bf16(normal(np.random.default_rng(98), 3, 2, 64))
    for pool in (4, 0):
        plan = fa.Plan.mx_plan(8, 2, 64, [0, 2, 3], [300, 129], m.cap, m.cap, n_pool_tiles=pool)
        out, lse = m.outs()
        with pytest.raises(fa.FkaError, match="need 5 tiles, the plan's n_pool_tiles is"):
            plan.decode_mx(out=out, out_lse=lse, **m.dev)
        with pytest.raises(fa.FkaError, match="need 5 tiles"):
            plan.step_mx(m.dev["q"], kn, kn, m.tiles, m.dev["suffix_k"], m.dev["suffix_v"], m.dev["suffix_len"], out, lse)
        torch.cuda.synchronize()
        assert torch.isnan(out).all() and np.array_equal(m.dev["suffix_len"].cpu().numpy(), m.lens) and plan.device_error() == 0
    plan = fa.Plan.mx_plan(8, 2, 64, [0, 2, 3], [300, 300], m.cap, m.cap, n_pool_tiles=5)  # two forks of one prefix
    m.prefixes, m.pk[1], m.pv[1] = [300, 300], m.pk[0], m.pv[0]
    out, lse = m.outs()
    plan.decode_mx(out=out, out_lse=lse, tile_table=dev_i32([[0, 1, 2], [0, 1, 2]]), **m.dev)
    m.check(out.cpu().numpy(), lse.cpu().numpy(), "a shared prefix")
    assert plan.device_error() == 0


def test_rotate_buffers_side_by_side(fa):  # noqa: F811
    """Buffers that touch, q_out in a gap between two tokens' rows, and q_out at a dense q are not overlaps: the results are those of
    buffers apart."""
    rng = np.random.default_rng(99)
    n, hq, hkv, d = 2, 4, 2, 64
    width, qn, kn = (hq + 2 * hkv) * d, n * hq * d, hkv * n * d
    step = width + qn + 2 * kn
    rows = normal(rng, n, width)
    arena = torch.zeros(2 * step, dtype=torch.bfloat16, device="cuda")
    tok = arena[: n * step].view(1, n, step)
    tok[..., :width] = dev_bf16(rows)
    part = lambda t, a, b: t[..., a * d: b * d].unflatten(-1, (-1, d))  # noqa: E731
    pos, freq = dev_i32([[5, 6]]), torch.full((32,), 0.7, dtype=torch.float64, device="cuda")

    def run(t, q_out, kc, vc):
        fa.rotate_append(part(t, 0, hq), part(t, hq, hq + hkv), part(t, hq + hkv, hq + 2 * hkv), pos, freq, q_out, kc, vc)
        return [host(x) for x in (q_out, kc, vc)]

    apart = [torch.empty(1, n, hq, d, dtype=torch.bfloat16, device="cuda")] + [
        torch.empty(1, hkv, n, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    want = run(dev_bf16(rows).view(1, n, width), *apart)
    gap = arena[width: step]  # between the first token's row and the second's
    got = run(tok, gap[:qn].view(1, n, hq, d), gap[qn: qn + kn].view(1, hkv, n, d), gap[qn + kn:].view(1, hkv, n, d))
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    assert np.array_equal(host(tok[0, :, :width]), rows), "what was read is as it was"
    q = dev_bf16(rows)[None, :, : hq * d].contiguous().view(1, n, hq, d)
    t = dev_bf16(rows).view(1, n, width)
    fa.rotate_append(q, part(t, hq, hq + hkv), part(t, hq + hkv, hq + 2 * hkv), pos, freq, q, *apart[1:])
    assert np.array_equal(host(q), want[0])


@pytest.mark.parametrize("d,inter,tokens", [(64, False, 12), (128, True, 12), (128, False, 2052)])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-35])
def test_rotate_norms_heads_of_every_magnitude(fa, eps, d, inter, tokens):  # noqa: F811
    """Heads from bf16's smallest numbers to its largest, beside ordinary ones in the same wave, are normed as the formula says, though
    their squares leave fp32's range."""
    rng = np.random.default_rng(101)
    hq, hkv = 11, 3
    exps = np.array([0, 127, 64, -64, -133, 100, -40, 0, -120, 63, -70])
    x = rng.uniform(0.5, 1, (1, tokens, hq, d)) * rng.choice([-1, 1], (1, tokens, hq, d)) * 2.0 ** exps[None, None, :, None]
    rows = bits_of(np.concatenate([x, x[:, :, 1:4], x[:, :, 4:7]], 2))
    rows[0, 0, 0, 1:] = 0  # one channel only
    w = bits_of(1 + 0.3 * rng.standard_normal(d))
    freq, pos = 1e4 ** (-np.arange(0, d, 2) / d), np.arange(tokens)[None]
    t = dev_bf16(rows)
    q_out = torch.empty(1, tokens, hq, d, dtype=torch.bfloat16, device="cuda")
    kc, vc = (torch.empty(1, hkv, tokens, d, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    fa.rotate_append(t[:, :, :hq], t[:, :, hq: hq + hkv], t[:, :, hq + hkv:], dev_i32(pos), torch.from_numpy(freq).cuda(), q_out, kc, vc,
                     q_weight=dev_bf16(w), k_weight=dev_bf16(w), eps=eps, interleaved=inter)
    e32 = float(np.float32(eps))
    for got, a, b in ((host(q_out), 0, hq), (host(kc).transpose(0, 2, 1, 3), hq, hq + hkv)):
        close_rotated(got, ref_rotate(value(rows[:, :, a:b]), value(w), pos.astype(float), freq, d, inter, e32), (eps, a))
    assert np.array_equal(host(vc).transpose(0, 2, 1, 3), rows[:, :, hq + hkv:])


def test_copies_past_4_gib(fa):  # noqa: F811
    """Pack, unpack and evict where the last head's rows, and a tile's id, lie past 32 bits of bytes: as from small buffers."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    rng = np.random.default_rng(110)
    hkv, d, n, cap, pool = 8, 128, 20000, 2_400_000, 32000
    assert (hkv - 1) * cap * d * 2 > 1 << 32 and (pool - 1) * hkv * 136 * d > 1 << 32
    small = [dev_bf16(normal(rng, hkv, n, d)) for _ in "kv"]
    big = [torch.empty(hkv, cap, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    for b, s in zip(big, small):
        b[:, :n] = s
    # evict
    w = rng.random((hkv, n)).astype(np.float32)
    keep, weights = 700, torch.from_numpy(w).cuda()
    index = torch.empty(hkv, keep, dtype=torch.int32, device="cuda")
    ko, vo = (torch.empty(hkv, keep, d, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    fa.evict(*big, weights, index, ko, vo, n_first=3, n_last=5, length=n, workspace=fa.evict_workspace(hkv, n))
    want = ref_evict(w, keep, 3, 5)
    assert np.array_equal(index.cpu().numpy(), want)
    for got, s in zip((ko, vo), small):
        assert np.array_equal(host(got), host(s)[np.arange(hkv)[:, None], want])
    # pack and unpack
    m = 300
    row = [pool - 1, 7, pool - 2]
    tiles = torch.empty(pool, hkv, 136 * d, dtype=torch.uint8, device="cuda")
    fa.mx_pack(*big, tiles, tile_row=dev_i32(row), length=m)
    near = torch.empty(3, hkv, 136 * d, dtype=torch.uint8, device="cuda")
    fa.mx_pack(*[s[:, :m].contiguous() for s in small], near)
    for i, r in enumerate(row):
        assert torch.equal(tiles[r], near[i])
    back = [torch.empty(hkv, m, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    fa.mx_unpack(near, *back)
    for b in big:
        b[:, : m + 1] = 7.0
    fa.mx_unpack(tiles, *big, tile_row=dev_i32(row), length=m)
    for b, s in zip(big, back):
        assert torch.equal(b[:, :m], s) and (b[:, m] == 7.0).all()
