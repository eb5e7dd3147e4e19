"""Edges of the operators around a snapshot's cache on the GPU: values, magnitudes and sizes at which a result is easily lost.
Tolerances as in tests/test_gpu_cache_ops.py, or derived beside the test."""
import numpy as np
import pytest
import torch

from tests.gpu_util import dev_bf16, dev_i32
from tests.test_gpu_cache_ops import Mx, fa, host, normal, value  # noqa: F401  (fa is the fixture)

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
