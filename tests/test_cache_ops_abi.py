"""Refusals of the operators around a snapshot's cache (rotate_append, mx_*, key_weights, evict): host validation
before any HIP call, and the binding's checks of the tensors (no GPU needed)."""
import ctypes as C

import pytest
import torch

P = C.c_void_p(4096)       # an aligned address that a refused call never follows
ODD = C.c_void_p(4096 + 4)


@pytest.fixture(scope="module")
def fa():
    from paper_2608_13667_amd import forkattn
    return forkattn


def _rotate(fa, paged=False, q=P, freq=P, weight=None, cache=P, cap=64, lens=P, pages=4, **over):
    d = dict(n_seqs=5, n_tokens=1, n_q_heads=8, n_kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, max_len=64, advance=0,
             eps=1e-6, q_stride=768, k_stride=768, v_stride=768)
    d.update(over)
    desc = fa.RotateDesc(*d.values())
    if paged:
        return fa.raw_call("fka_rotate_append_paged", C.byref(desc), q, P, P, weight, None, freq, P, P, cache, P, P, P, pages, 100,
                           lens, None, None)
    return fa.raw_call("fka_rotate_append", C.byref(desc), q, P, P, weight, None, freq, P, P, cache, P, cap, lens, None, None)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("over,status,needle", [
    (dict(n_seqs=0), -1, "n_seqs"), (dict(n_tokens=0), -1, "n_tokens"), (dict(n_kv_heads=0), -1, "head counts"),
    (dict(head_dim=96), -2, "head_dim"), (dict(rotary_dim=24), -2, "rotary_dim"), (dict(rotary_dim=80), -1, "rotary_dim"),
    (dict(rotary_dim=-16), -1, "rotary_dim"), (dict(interleaved=2), -1, "interleaved"), (dict(advance=2), -1, "advance"),
    (dict(advance=1, lens=None), -1, "suffix_len"), (dict(eps=float("nan")), -1, "eps"), (dict(eps=-1.0), -1, "eps"),
    (dict(max_len=-1), -1, "max_len"), (dict(q_stride=511), -1, "stride"), (dict(k_stride=132), -1, "multiples"),
    (dict(v_stride=64), -1, "stride"), (dict(n_seqs=2**20, n_tokens=64), -2, "tokens"), (dict(q=None), -1, "q is null"),
    (dict(q=ODD), -1, "aligned"), (dict(weight=ODD), -1, "weight"), (dict(freq=None), -1, "freq"), (dict(freq=ODD), -1, "freq"),
    (dict(cache=None), -1, "null"), (dict(max_len=2**31 - 1, cap=2**31 - 1), -2, "too long"),
])
def test_rotate_rejects(fa, paged, over, status, needle):
    assert _rotate(fa, paged, **over) == status
    assert needle in fa.last_error()


def test_rotate_rejects_layouts(fa):
    assert _rotate(fa, cap=63) == -1 and "suffix_cap" in fa.last_error()
    assert _rotate(fa, True, pages=0) == -1 and "max_pages" in fa.last_error()
    n = None
    assert fa.raw_call("fka_rotate_append", n, n, n, n, n, n, n, n, n, n, n, 4, n, n, n) == -1


@pytest.mark.parametrize("name", ["fka_mx_pack", "fka_mx_unpack"])
@pytest.mark.parametrize("over,status,needle", [
    (dict(hkv=0), -1, "n_kv_heads"), (dict(d=96), -2, "head_dim"), (dict(frm=-128), -1, "from"), (dict(length=-1), -1, "from"),
    (dict(frm=256), -1, "from"), (dict(cap=199), -1, "cap"), (dict(n=1), -1, "tiles"), (dict(n=-1), -1, "n_pool_tiles"),
    (dict(k=None), -1, "null"), (dict(tiles=ODD), -1, "aligned"), (dict(length=2**31 - 1, n=2**30, cap=2**31 - 1), -2, "many"),
])
def test_mx_copies_reject(fa, name, over, status, needle):
    a = dict(hkv=2, d=64, frm=0, length=200, cap=200, n=2, k=P, tiles=P)
    a.update(over)
    if name == "fka_mx_pack":
        st = fa.raw_call(name, a["hkv"], a["d"], a["frm"], a["length"], a["k"], P, a["cap"], a["tiles"], None, a["n"], None, None)
    else:
        st = fa.raw_call(name, a["hkv"], a["d"], a["frm"], a["length"], a["tiles"], None, a["n"], a["k"], P, a["cap"], None, None)
    assert st == status and needle in fa.last_error()


def test_mx_pack_writes_whole_tiles_only(fa):
    assert fa.raw_call("fka_mx_pack", 2, 64, 100, 200, P, P, 100, P, None, 2, None, None) == -1 and "multiple" in fa.last_error()
    assert fa.raw_call("fka_mx_pack", 2, 64, 128, 128, None, None, 0, None, None, 2, None, None) == 0  # nothing to do
    assert fa.mx_tile_bytes(8, 128) == 8 * 136 * 128 and fa.mx_tile_bytes(8, 96) == 0 and fa.mx_tile_bytes(0, 64) == 0


def _plan_mx(fa, gs=(0, 5), gl=(300,), heads=(8, 2, 64), **over):
    import numpy as np
    d = dict(n_seqs=5, n_groups=1, max_tiles_per_group=3, n_pool_tiles=3, suffix_cap=64, max_suffix_len=64, blocks=0)
    d.update(over)
    h, desc, out = fa.Heads(*heads, 0.0), fa.MxDesc(*d.values()), C.c_void_p()
    gs, gl = np.array(gs, np.int32), np.array(gl, np.int32)
    st = fa.raw_call("fka_plan_create_mx", C.byref(h), C.byref(desc), gs.ctypes.data_as(C.c_void_p),
                     gl.ctypes.data_as(C.c_void_p), C.byref(out))
    assert not out.value
    return st


@pytest.mark.parametrize("over,status,needle", [
    (dict(heads=(8, 3, 64)), -1, "multiple"), (dict(heads=(8, 2, 96)), -2, "head_dim"), (dict(n_seqs=0, gs=(0, 0)), -1, "n_seqs"),
    (dict(max_tiles_per_group=2), -1, "needs 3 tiles"), (dict(max_tiles_per_group=0), -1, "max_tiles"),
    (dict(n_pool_tiles=-1), -1, "n_pool_tiles"), (dict(suffix_cap=0), -1, "suffix_cap"), (dict(max_suffix_len=65), -1, "max_suffix_len"),
    (dict(blocks=-1), -1, "blocks"), (dict(gs=(0, 4)), -1, "group_start"), (dict(gs=(1, 5)), -1, "group_start"),
    (dict(n_groups=2, gs=(0, 0, 5), gl=(1, 1)), -1, "empty"), (dict(gl=(-1,)), -1, "negative"), (dict(n_seqs=513, gs=(0, 513)), -2, "513"),
    (dict(heads=(32, 2, 64)), -2, "rows"), (dict(gl=(2**31 - 1,), max_tiles_per_group=2**30), -2, "too long"),
    (dict(n_groups=6), -2, "groups"), (dict(suffix_cap=2**31 - 1, max_suffix_len=2**31 - 1), -2, "too long"),
    (dict(n_groups=2, gs=(0, -5, 5), gl=(1, 1)), -1, "empty"),
])
def test_mx_plan_rejects(fa, over, status, needle):
    assert _plan_mx(fa, **over) == status
    assert needle in fa.last_error()


def test_mx_calls_reject_a_null_plan(fa):
    assert fa.raw_call("fka_fork_decode_mx", *[None] * 10) == -1
    assert fa.raw_call("fka_fork_step_mx", *[None] * 12) == -1


@pytest.mark.parametrize("over,status,needle", [
    (dict(heads=(8, 3, 64)), -1, "multiple"), (dict(heads=(8, 2, 80)), -2, "head_dim"), (dict(rows=-1), -1, "n_rows"),
    (dict(length=-1), -1, "len"), (dict(kcap=99), -1, "k_cap"), (dict(wcap=99), -1, "weights_cap"), (dict(decay=-0.5), -1, "decay"),
    (dict(decay=float("inf")), -1, "decay"), (dict(q=None), -1, "q is null"), (dict(q=ODD), -1, "aligned"), (dict(k=ODD), -1, "aligned"),
    (dict(rows=2**30), -2, "many"),
])
def test_key_weights_reject(fa, over, status, needle):
    a = dict(heads=(8, 2, 64), rows=5, length=100, q=P, k=P, kcap=100, wcap=100, decay=0.5)
    a.update(over)
    h = fa.Heads(*a["heads"], 0.0)
    st = fa.raw_call("fka_key_weights", C.byref(h), a["rows"], a["length"], a["q"], P, a["k"], a["kcap"], P, a["wcap"], a["decay"], None)
    assert st == status and needle in fa.last_error()


@pytest.mark.parametrize("over,status,needle", [
    (dict(hkv=0), -1, "n_kv_heads"), (dict(d=32), -2, "head_dim"), (dict(keep=101), -1, "keep"), (dict(keep=-1), -1, "keep"),
    (dict(first=41), -1, "n_first"), (dict(first=-1), -1, "n_first"), (dict(first=2**31 - 1, last=2**31 - 1), -1, "n_first"),
    (dict(cap=99), -1, "kv_cap"), (dict(wcap=99), -1, "weights_cap"), (dict(k=ODD), -1, "aligned"), (dict(k=None), -1, "null"),
    (dict(work=None), -1, "workspace"), (dict(bytes=100), -1, "workspace"),
])
def test_evict_rejects(fa, over, status, needle):
    a = dict(hkv=2, d=64, length=100, keep=50, first=4, last=10, k=P, cap=100, wcap=100, work=P, bytes=1 << 20)
    a.update(over)
    st = fa.raw_call("fka_evict", a["hkv"], a["d"], a["length"], a["keep"], a["first"], a["last"], a["k"], P, a["cap"], P, a["wcap"],
                     P, P, P, None, a["work"], a["bytes"], None)
    assert st == status and needle in fa.last_error()


@pytest.mark.parametrize("name", ["index", "k_out", "v_out", "weights_out", "work"])
def test_evict_rejects_overlaps(fa, name):
    """Each of what it writes against each other range, overlapping by a few bytes at either end; ranges that only touch would pass."""
    hkv, d, n, cap, keep = 2, 64, 100, 128, 50
    size = dict(k=(cap + n) * d * 2, v=(cap + n) * d * 2, weights=(cap + n) * 4, index=hkv * keep * 4, k_out=hkv * keep * d * 2,
                v_out=hkv * keep * d * 2, weights_out=hkv * keep * 4, work=fa.raw_call("fka_evict_bytes", hkv, n))
    for other in size:
        if other == name:
            continue
        for shift in (16 - size[name] + size[name] % 16, (size[other] - 16) // 16 * 16, 0):
            at = {x: (1 << 30) + (i << 24) for i, x in enumerate(size)}
            at[name] = at[other] + shift
            p = {x: C.c_void_p(y) for x, y in at.items()}
            st = fa.raw_call("fka_evict", hkv, d, n, keep, 4, 10, p["k"], p["v"], cap, p["weights"], cap, p["index"], p["k_out"],
                             p["v_out"], p["weights_out"], p["work"], size["work"], None)
            assert st == -1 and "overlaps" in fa.last_error() and name.replace("work", "workspace") in fa.last_error(), (other, shift)


def test_evict_sizes(fa):
    lib = fa._lib
    assert lib.fka_evict_bytes(0, 5) == 0 and lib.fka_evict_bytes(2, -1) == 0
    assert lib.fka_evict_bytes(8, 131072) >= 3 * 8 * 2048 * 4
    assert fa.raw_call("fka_evict", 2, 64, 100, 0, 0, 0, None, None, 100, None, 100, None, None, None, None, None, 0, None) == 0


def test_binding_checks_tensors(fa):
    """Shapes, types, strides and the device are refused before any call."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q, k, cache = bf(2, 1, 8, 64), bf(2, 1, 2, 64), bf(2, 2, 16, 64)
    pos, freq = torch.zeros(2, 1, dtype=torch.int32), torch.ones(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="GPU"):
        fa.rotate_append(q, k, k, pos, freq, q, cache, cache)
    with pytest.raises(ValueError, match="dense"):
        fa.rotate_append(bf(2, 1, 64, 8).transpose(2, 3), k, k, pos, freq, q, cache, cache)
    with pytest.raises(ValueError, match="evenly"):
        fa.rotate_append(bf(2, 6, 8, 64)[:, :3], bf(2, 3, 2, 64), bf(2, 3, 2, 64), pos, freq, bf(2, 3, 8, 64), cache, cache)
    with pytest.raises(ValueError, match="Hkv"):
        fa.rotate_append(q, k, bf(2, 1, 1, 64), pos, freq, q, cache, cache)
    with pytest.raises(ValueError, match="cap"):
        fa.rotate_append(q, k, k, pos, freq, q, bf(1, 2, 16, 64), cache)
    with pytest.raises(ValueError, match="q_out"):
        fa.rotate_append(q, k, k, pos[:1], freq, q, cache, cache)
    with pytest.raises(ValueError, match="suffix_len"):
        fa.rotate_append(q, k, k, pos, freq, q, cache, cache, torch.zeros(3, dtype=torch.int32))
    tiles = torch.zeros(2, 2, 136 * 64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        fa.mx_pack(bf(2, 200, 64), bf(2, 200, 64), tiles)
    with pytest.raises(ValueError, match="tiles"):
        fa.mx_pack(bf(2, 200, 64), bf(2, 200, 64), tiles[:, :1])
    with pytest.raises(ValueError, match="tile_row"):
        fa.mx_pack(bf(2, 200, 64), bf(2, 200, 64), tiles, tile_row=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="lse"):
        fa.key_weights(bf(3, 8, 64), torch.zeros(2, 8), bf(2, 9, 64), torch.zeros(2, 9))
    with pytest.raises(ValueError, match="keep"):
        fa.evict(bf(2, 9, 64), bf(2, 9, 64), torch.zeros(2, 9), torch.zeros(2, 4, dtype=torch.int32), bf(2, 5, 64), bf(2, 4, 64),
                 workspace=None)
    with pytest.raises(ValueError, match="group_prefix_len"):
        fa.Plan.mx_plan(8, 2, 64, [0, 5], [1, 2], 64, 64, n_pool_tiles=1)


def _rotate_at(fa, paged, at, sizes):
    """A rotate call with every buffer at an address of its own; nothing is launched where it is refused."""
    n, cap, pages = sizes
    desc = fa.RotateDesc(3, n, 4, 2, 64, 64, 0, cap, 0, 1e-6, 768, 768, 768)
    p = {x: C.c_void_p(y) for x, y in at.items()}
    head = [C.byref(desc), p["q"], p["k"], p["v"], p["q_weight"], p["k_weight"], p["freq"], p["positions"], p["q_out"], p["the K cache"],
            p["the V cache"]]
    if paged:
        return fa.raw_call("fka_rotate_append_paged", *head, p["page_table"], p["prefix_len"], 4, pages, p["suffix_len"], p["err"], None)
    return fa.raw_call("fka_rotate_append", *head, cap, p["suffix_len"], p["err"], None)


@pytest.mark.parametrize("name", ["q_out", "the K cache", "the V cache"])
@pytest.mark.parametrize("paged", [False, True])
def test_rotate_rejects_overlaps(fa, paged, name):
    """Each of what it writes against each other buffer, by a few bytes at either end; q, k and v by their rows, the last one too."""
    n, cap, pages = 5, 16, 7
    tokens, row = 3 * n, 768 * 2
    cache = (pages * 16 if paged else 3 * cap) * 2 * 64 * 2
    size = {"q": 4 * 128, "k": 2 * 128, "v": 2 * 128, "q_weight": 128, "k_weight": 128, "freq": 256, "positions": tokens * 4,
            "suffix_len": 12, "err": 4, "q_out": tokens * 4 * 128, "the K cache": cache, "the V cache": cache}
    if paged:
        size.update(page_table=3 * 4 * 4, prefix_len=12)
    for other in size:
        if other == name:
            continue
        for r in (0, 1, tokens - 1) if other in "qkv" else (0,):
            for shift in (16 - size[name], (size[other] - 1) // 16 * 16, 0):
                at = {x: (1 << 30) + (i << 24) for i, x in enumerate(size)}
                at[name] = at[other] + r * row + shift
                assert _rotate_at(fa, paged, at, (n, cap, pages)) == -1, (other, r, shift)
                # (a row's neighbours may be met first)
                assert f"{name} overlaps {other}" in fa.last_error() or f"{other} overlaps {name}" in fa.last_error(), fa.last_error()


def test_rotate_q_out_is_q_or_apart(fa):
    """q_out at q's own address is refused where q's rows have gaps, in which q_out's rows would lie."""
    size = ["q", "k", "v", "q_weight", "k_weight", "freq", "positions", "suffix_len", "err", "q_out", "the K cache", "the V cache"]
    at = {x: (1 << 30) + (i << 24) for i, x in enumerate(size)}
    at["q_out"] = at["q"]
    assert _rotate_at(fa, False, at, (1, 16, 0)) == -1 and "q_out overlaps q" in fa.last_error()


def _places(size):
    return {x: (1 << 30) + (i << 24) for i, x in enumerate(size)}


def _each_overlap(size, names):
    """Addresses with one of `names` upon another buffer, by a few bytes at either end."""
    for name in names:
        for other in size:
            for shift in (16 - (size[name] + 15) // 16 * 16, (size[other] - 1) // 16 * 16, 0):
                if other != name:
                    at = _places(size)
                    at[name] = at[other] + shift
                    yield name, other, {x: C.c_void_p(y) for x, y in at.items()}


def test_mx_copies_reject_overlaps(fa):
    hkv, d, n, cap, pool = 2, 64, 200, 230, 3
    side = (cap + n) * d * 2
    size = dict(k=side, v=side, tiles=pool * hkv * 136 * d, tile_row=8, err=4)
    for name, other, p in _each_overlap(size, ["tiles"]):
        st = fa.raw_call("fka_mx_pack", hkv, d, 0, n, p["k"], p["v"], cap, p["tiles"], p["tile_row"], pool, p["err"], None)
        assert st == -1 and f"{name} overlaps {other}" in fa.last_error(), (name, other)
    for name, other, p in _each_overlap(size, ["k", "v"]):
        st = fa.raw_call("fka_mx_unpack", hkv, d, 0, n, p["tiles"], p["tile_row"], pool, p["k"], p["v"], cap, p["err"], None)
        assert st == -1 and "overlaps" in fa.last_error() and {name, other} == set(fa.last_error().split(" overlaps ")), (name, other)


def test_key_weights_reject_overlaps(fa):
    h, rows, n, kcap, wcap = fa.Heads(8, 2, 64, 0.0), 5, 100, 130, 120
    size = dict(weights=(wcap + n) * 4, q=rows * 8 * 64 * 2, lse=rows * 8 * 4, k=(kcap + n) * 64 * 2)
    for name, other, p in _each_overlap(size, ["weights"]):
        st = fa.raw_call("fka_key_weights", C.byref(h), rows, n, p["q"], p["lse"], p["k"], kcap, p["weights"], wcap, 0.5, None)
        assert st == -1 and f"weights overlaps {other}" in fa.last_error(), (other, fa.last_error())


@pytest.mark.parametrize("hkv,length", [(65535, 100), (2, 2**30), (65536, 100), (2**31 - 1, 100), (2, 2**30 + 1), (2, 2**31 - 1), (0, 9), (2, -1)])
def test_evict_bytes_are_zero_where_evict_refuses(fa, hkv, length):
    st = fa.raw_call("fka_evict", hkv, 64, length, 0, 0, 0, None, None, length, None, length, None, None, None, None, None, 0, None)
    assert (st == 0) == (fa._lib.fka_evict_bytes(hkv, length) > 0), (st, fa.last_error())
