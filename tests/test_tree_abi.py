"""Refusals of the operators of drafted trees (tree_layout, tree_attend, tree_accept): host validation before any HIP
call, and the binding's checks of the tensors (no GPU needed)."""
import ctypes as C

import pytest
import torch

ODD = C.c_void_p((1 << 40) + 2)
_at = [1 << 40]


def _ptr(size=1 << 30):
    """An aligned address with room behind it that no other has; a refused call never follows it."""
    _at[0] += size
    return C.c_void_p(_at[0] - size)


@pytest.fixture(scope="module")
def fa():
    from paper_2608_13667_amd import forkattn
    return forkattn


def _layout(fa, N=3, n=4, **over):
    a = dict(parents=_ptr(), base=_ptr(), masks=_ptr(), positions=_ptr(), err=None)
    a.update(over)
    return fa.raw_call("fka_tree_layout", N, n, *a.values(), None)


@pytest.mark.parametrize("over,status,needle", [
    (dict(N=0), -1, "n_branches"), (dict(n=0), -1, "n_nodes"), (dict(n=65), -2, "64"), (dict(N=2**20 + 1), -2, "trees"),
    (dict(parents=None), -1, "parents is null"), (dict(base=ODD), -1, "base is not"), (dict(masks=None), -1, "masks is null"),
    (dict(masks=C.c_void_p((1 << 40) + 4)), -1, "8-byte"), (dict(positions=None), -1, "positions"), (dict(err=ODD), -1, "err"),
])
def test_layout_rejects(fa, over, status, needle):
    assert _layout(fa, **over) == status
    assert needle in fa.last_error()


def test_layout_rejects_overlaps(fa):
    p = _ptr()
    for over, needle in ((dict(masks=p, positions=C.c_void_p(p.value + 8)), "overlaps positions"),
                         (dict(parents=p, masks=C.c_void_p(p.value + 40)), "overlaps parents"),
                         (dict(base=p, positions=C.c_void_p(p.value + 8)), "overlaps base"), (dict(err=p, positions=p), "overlaps err")):
        assert _layout(fa, **over) == -1
        assert needle in fa.last_error()


def _plan(fa, name, heads=(8, 2, 64), **over):
    d = dict(n_branches=2, n_tokens=4, prefix_len=100, suffix_cap=64, max_suffix_len=64, blocks=0)
    if name.endswith("paged"):
        d = dict(n_branches=2, n_tokens=4, prefix_len=100, page_size=16, max_pages_per_seq=11, n_pool_pages=30, max_suffix_len=64, blocks=0)
    d.update(over)
    h, out = fa.Heads(*heads, 0.0), C.c_void_p()
    desc = (fa.PrefillPagedDesc if name.endswith("paged") else fa.PrefillDesc)(*d.values())
    st = fa.raw_call(name, C.byref(h), C.byref(desc), C.byref(out))
    assert not out.value
    return st


@pytest.mark.parametrize("name", ["fka_plan_create_tree", "fka_plan_create_tree_paged"])
@pytest.mark.parametrize("over,status,needle", [
    (dict(n_branches=0), -1, "n_branches"), (dict(n_tokens=0), -1, "n_tokens"), (dict(n_tokens=65, max_suffix_len=65), -2, "64"),
    (dict(n_branches=129), -2, "512"), (dict(prefix_len=-1), -1, "prefix_len"), (dict(max_suffix_len=3), -1, "max_suffix_len"),
    (dict(blocks=-1), -1, "blocks"), (dict(heads=(8, 3, 64)), -1, "multiple"), (dict(heads=(8, 2, 96)), -2, "head_dim"),
    (dict(heads=(65, 1, 64)), -2, "query heads"),
])
def test_plans_reject(fa, name, over, status, needle):
    if name == "fka_plan_create_tree" and over.get("max_suffix_len") == 65:
        over = dict(over, suffix_cap=65)
    if name.endswith("paged") and over.get("max_suffix_len") == 65:
        over = dict(over, max_pages_per_seq=12)
    assert _plan(fa, name, **over) == status
    assert needle in fa.last_error()


def test_plans_reject_layouts(fa):
    assert _plan(fa, "fka_plan_create_tree", suffix_cap=63) == -1 and "suffix_cap" in fa.last_error()
    assert _plan(fa, "fka_plan_create_tree_paged", page_size=32) == -1 and "page_size" in fa.last_error()
    assert _plan(fa, "fka_plan_create_tree_paged", max_pages_per_seq=10) == -1 and "pages" in fa.last_error()
    n = None
    assert fa.raw_call("fka_tree_attend", *[n] * 11) == -1 and "plan is null" in fa.last_error()
    assert fa.raw_call("fka_tree_attend_paged", *[n] * 10) == -1 and "plan is null" in fa.last_error()


def _accept(fa, paged=False, cap=64, pages=4, pool=100, **over):
    d = dict(n_branches=3, n_nodes=8, n_kv_heads=2, head_dim=64, max_len=64, advance=1)
    a = dict(parents=_ptr(), masks=_ptr(), tokens=_ptr(), targets=_ptr(), k=_ptr(), v=_ptr(), table=_ptr(), prefix=_ptr(), lens=_ptr(),
             path=_ptr(), count=_ptr(), next=_ptr(), err=None)
    for key, x in over.items():
        (d if key in d else a)[key] = x
    desc = fa.AcceptDesc(*d.values())
    tree = [a[x] for x in ("parents", "masks", "tokens", "targets", "k", "v")]
    end = [a[x] for x in ("lens", "path", "count", "next", "err")]
    if paged:
        return fa.raw_call("fka_tree_accept_paged", C.byref(desc), *tree, a["table"], a["prefix"], pages, pool, *end, None)
    return fa.raw_call("fka_tree_accept", C.byref(desc), *tree, cap, *end, None)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("over,status,needle", [
    (dict(n_branches=0), -1, "n_branches"), (dict(n_nodes=0), -1, "n_nodes"), (dict(n_nodes=65), -2, "64"),
    (dict(n_branches=2**20 + 1), -2, "trees"), (dict(n_kv_heads=0), -1, "n_kv_heads"), (dict(head_dim=80), -2, "head_dim"),
    (dict(max_len=-1), -1, "max_len"), (dict(max_len=2**31 - 1, cap=2**31 - 1), -2, "too long"), (dict(advance=2), -1, "advance"),
    (dict(parents=None), -1, "parents"), (dict(masks=ODD), -1, "masks"), (dict(tokens=None), -1, "tokens"), (dict(targets=ODD), -1, "targets"),
    (dict(k=None), -1, "cache"), (dict(v=C.c_void_p((1 << 40) + 8)), -1, "cache"), (dict(lens=None), -1, "suffix_len"),
    (dict(path=None), -1, "path"), (dict(count=None), -1, "count"), (dict(next=ODD), -1, "next"), (dict(err=ODD), -1, "err"),
])
def test_accept_rejects(fa, paged, over, status, needle):
    assert _accept(fa, paged, **over) == status
    assert needle in fa.last_error()


def test_accept_rejects_layouts_and_overlaps(fa):
    assert _accept(fa, cap=63) == -1 and "suffix_cap" in fa.last_error()
    assert _accept(fa, True, pages=0) == -1 and "max_pages" in fa.last_error()
    assert _accept(fa, True, table=None) == -1 and "page_table" in fa.last_error()
    assert _accept(fa, True, prefix=None) == -1 and "prefix_len" in fa.last_error()
    assert fa.raw_call("fka_tree_accept", *[None] * 7, 4, *[None] * 6) == -1 and "desc" in fa.last_error()
    p = _ptr()
    q = C.c_void_p(p.value + 16)
    for over, needle in ((dict(k=p, v=q), "overlaps the V cache"), (dict(path=p, count=q), "overlaps count"),
                         (dict(tokens=p, path=q), "overlaps tokens"), (dict(lens=p, next=p), "overlaps suffix_len"),
                         (dict(masks=p, k=q), "overlaps masks")):
        for paged in (False, True):
            assert _accept(fa, paged, **over) == -1
            assert needle in fa.last_error()
    assert _accept(fa, True, table=p, v=q) == -1 and "page_table" in fa.last_error()


def test_binding_checks_shapes(fa):
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    m = lambda *s: torch.zeros(s, dtype=torch.int64)  # noqa: E731
    kv = torch.zeros(2, 1, 20, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="base"):
        fa.tree_layout(i(2, 4), i(3), m(2, 4), i(2, 4))
    with pytest.raises(ValueError, match="masks"):
        fa.tree_layout(i(2, 4), i(2), m(2, 5), i(2, 4))
    with pytest.raises(ValueError, match="on the GPU"):
        fa.tree_layout(i(2, 4), i(2), m(2, 4), i(2, 4))
    with pytest.raises(ValueError, match="targets"):
        fa.tree_accept(i(2, 4), m(2, 4), i(2, 4), i(2, 3), kv, kv, i(2), i(2, 4), i(2), i(2))
    with pytest.raises(ValueError, match="count"):
        fa.tree_accept(i(2, 4), m(2, 4), i(2, 4), i(2, 4), kv, kv, i(2), i(2, 4), i(1), i(2))
    with pytest.raises(ValueError, match="on the GPU"):
        fa.tree_accept(i(2, 4), m(2, 4), i(2, 4), i(2, 4), kv, kv, i(2), i(2, 4), i(2), i(2))


def _sample(fa, R=3, V=100, bf16=0, stride=100, work=1 << 20, **over):
    a = dict(logits=_ptr(), temperature=_ptr(), top_k=_ptr(), top_p=_ptr(), min_p=_ptr(), u=_ptr(), tokens=_ptr(), logprob=_ptr(), err=None,
             workspace=_ptr())
    a.update(over)
    desc = fa.SampleDesc(R, V, bf16, stride)
    return fa.raw_call("fka_sample", C.byref(desc), *a.values(), work, None)


@pytest.mark.parametrize("over,status,needle", [
    (dict(R=-1), -1, "n_rows"), (dict(V=0), -1, "n_vocab"), (dict(V=2**18 + 1, stride=2**19), -2, "logits"), (dict(R=2**17 + 1), -2, "rows"),
    (dict(bf16=2), -1, "bf16"), (dict(stride=99), -1, "logits_stride"), (dict(stride=-1), -1, "logits_stride"),
    (dict(logits=None), -1, "logits is null"), (dict(logits=ODD), -1, "logits is not 4-byte"), (dict(bf16=1, logits=C.c_void_p(4097)), -1, "2-byte"),
    (dict(u=None), -1, "u is null"), (dict(tokens=None), -1, "tokens"), (dict(temperature=ODD), -1, "temperature"), (dict(top_k=ODD), -1, "top_k"),
    (dict(top_p=ODD), -1, "top_p"), (dict(min_p=ODD), -1, "min_p"), (dict(logprob=ODD), -1, "logprob"), (dict(err=ODD), -1, "err"),
    (dict(workspace=None), -1, "workspace"), (dict(work=0), -1, "workspace of 0"),
])
def test_sample_rejects(fa, over, status, needle):
    assert _sample(fa, **over) == status
    assert needle in fa.last_error()


def test_sample_rejects_overlaps(fa):
    p = _ptr()
    q = C.c_void_p(p.value + 8)
    for over, needle in ((dict(tokens=p, logprob=q), "overlaps logprob"), (dict(u=p, tokens=q), "overlaps u"), (dict(logits=p, tokens=q), "overlaps logits"),
                         (dict(workspace=p, top_p=p), "overlaps top_p"), (dict(err=p, logprob=p), "overlaps err")):
        assert _sample(fa, **over) == -1
        assert needle in fa.last_error()
    assert fa.raw_call("fka_sample", *[None] * 11, 0, None) == -1 and "desc" in fa.last_error()
    assert fa.raw_call("fka_sample_bytes", -1, 5) == 0 and fa.raw_call("fka_sample_bytes", 5, 2**18 + 1) == 0
    assert fa.raw_call("fka_sample_bytes", 5, 2**18) > 0


def test_sample_binding_checks_shapes(fa):
    f = lambda *s: torch.zeros(s)  # noqa: E731
    i, w = torch.zeros(2, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="fp32 or bf16"):
        fa.sample(f(2, 5).half(), f(2), i, workspace=w)
    with pytest.raises(ValueError, match="dense"):
        fa.sample(f(5, 2).t(), f(2), i, workspace=w)
    with pytest.raises(ValueError, match="must be"):
        fa.sample(f(2, 5), f(3), i, workspace=w)
    with pytest.raises(ValueError, match="on the GPU"):
        fa.sample(f(2, 5), f(2), i, workspace=w)


def test_sample_workspace_of_a_larger_call_serves_a_smaller_one(fa):
    """The bytes fall neither with the rows nor with the vocabulary."""
    size = lambda r, v: fa.raw_call("fka_sample_bytes", r, v)  # noqa: E731
    many = sorted({*range(0, 1100), *(2**k + e for k in range(10, 17) for e in (-1, 0, 1)), 2**17})
    for v in (1, 100, 4097, 32000, 32768, 32769, 50000, 65536, 65537, 128000, 200003, 2**18):
        of = [size(r, v) for r in many]
        assert all(x > 0 for x in of)
        assert [(r, v) for r, x, y in zip(many[1:], of, of[1:]) if y < x] == []
    words = sorted({1, 2, *(at + e for at in range(4096, 2**18 + 1, 4096) for e in (-1, 0, 1) if at + e <= 2**18)})
    for r in (0, 1, 5, 63, 64, 65, 320, 819, 820, 1024, 1025, 5000, 2**17):
        of = [size(r, v) for v in words]
        assert [(r, v) for v, x, y in zip(words[1:], of, of[1:]) if y < x] == []


def test_sample_workspace_has_no_room_for_rows_that_are_not_shared(fa):
    """Up to 32768 logits a row's own block searches it: what is left are the tiles' sums and maxima and the groups' maxima, 12 bytes to 4096 logits and 4 to 16."""
    for r, v in ((320, 32000), (820, 32000), (5, 32768), (2**17, 1000)):
        assert fa.raw_call("fka_sample_bytes", r, v) <= r * (-(-v // 4096) * 12 + -(-v // 16) * 4) + 8 * 16
