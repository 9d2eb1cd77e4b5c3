"""Argument checks of the operators for several continuations of a prompt.  No GPU: every call returns from validation."""
import ctypes

import pytest
import torch

from paper_2405_03133_amd import binding as lb

F = 0x7F0000001000   # aligned, never dereferenced on these paths
B2, F4 = lb.LORY_BF16, lb.LORY_F32
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, OVERLAP = (lb.LORY_ERR_NULL, lb.LORY_ERR_SHAPE, lb.LORY_ERR_DTYPE, lb.LORY_ERR_ALIGN,
                                                 lb.LORY_ERR_WORKSPACE, lb.LORY_ERR_OVERLAP)


def beam_shape(**kw):
    d = dict(requests=3, beams=4, vocab=100, k=8, dtype=B2, row=100)
    d.update(kw)
    return lb.LoryBeamShape(**d)


BEAM = ("logits", "score", "score_out", "token", "parent", "workspace")


def beam(shape=None, bytes=1 << 40, **kw):
    a = {n: F + 0x100000 * i for i, n in enumerate(BEAM)}
    a.update(kw)
    return lb.lib().lory_beam_select(shape or beam_shape(), *a.values(), bytes, None)


@pytest.mark.parametrize("kw,rc", [(dict(requests=-1), SHAPE), (dict(beams=0), SHAPE), (dict(beams=65), SHAPE), (dict(vocab=0), SHAPE),
                                   (dict(vocab=(1 << 24) + 1, row=1 << 25), SHAPE), (dict(k=0), SHAPE), (dict(k=65), SHAPE), (dict(row=99), SHAPE),
                                   (dict(row=(1 << 36) + 1), SHAPE), (dict(requests=1 << 19), SHAPE), (dict(dtype=2), DTYPE)])
def test_beam_shapes(kw, rc):
    assert beam(beam_shape(**kw)) == rc
    assert lb.lib().lory_beam_select_workspace_bytes(beam_shape(**kw), ctypes.byref(ctypes.c_size_t())) == rc


def test_beam_arrays():
    assert lb.lib().lory_beam_select(None, *[F] * 6, 1 << 30, None) == NULL
    n = lb.lory_beam_select_workspace_bytes(beam_shape())
    assert beam(bytes=n - 1) == WORKSPACE
    assert lb.lib().lory_beam_select_workspace_bytes(beam_shape(), None) == NULL
    for name in BEAM:
        assert beam(**{name: None}) == NULL, name
        assert beam(**{name: F + 0x800000 + 1}) == ALIGN, name
    assert beam(beam_shape(dtype=F4), logits=F + 0x800000 + 2) == ALIGN and beam(workspace=F + 0x800000 + 8) == ALIGN
    addr = {m: F + 0x100000 * i for i, m in enumerate(BEAM)}
    for name in BEAM[2:]:
        for other in BEAM:
            if other != name:
                assert beam(**{name: addr[other]}) == OVERLAP, (name, other)
    # the last logit of the last row
    assert beam(beam_shape(row=1000), token=addr["logits"] + 2 * (11 * 1000 + 98)) == OVERLAP
    assert lb.lib().lory_beam_select(beam_shape(requests=0), *[None] * 6, 0, None) == lb.LORY_OK


def fork_shape(**kw):
    d = dict(old_rows=4, rows=6, width=8, page=16, pages=60, free_size=64, table_row=8, new_row=9)
    d.update(kw)
    return lb.LoryForkShape(**d)


FORK = ("lens", "src", "table", "free", "count", "lens_new", "table_new", "count_new", "copies", "status", "workspace")


def fork(shape=None, bytes=1 << 40, **kw):
    a = {n: F + 0x100000 * i for i, n in enumerate(FORK)}
    a.update(kw)
    return lb.lib().lory_kv_fork(shape or fork_shape(), *a.values(), bytes, None)


@pytest.mark.parametrize("kw", [dict(old_rows=-1), dict(old_rows=(1 << 20) + 1), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(width=0), dict(page=0),
                                dict(pages=0), dict(free_size=0), dict(table_row=7), dict(new_row=7), dict(new_row=(1 << 36) + 1),
                                dict(width=1 << 16, table_row=1 << 16, new_row=1 << 16, page=1 << 15)])
def test_fork_shapes(kw):
    assert fork(fork_shape(**kw)) == SHAPE
    assert lb.lib().lory_kv_fork_workspace_bytes(fork_shape(**kw), ctypes.byref(ctypes.c_size_t())) == SHAPE


def test_fork_arrays():
    assert lb.lib().lory_kv_fork(None, *[F] * 11, 1 << 30, None) == NULL
    for name in FORK:
        assert fork(**{name: None}) == NULL, name
        assert fork(**{name: F + 0x1000000 + 2}) == ALIGN, name
    addr = {n: F + 0x100000 * i for i, n in enumerate(FORK)}
    for name in FORK[3:]:
        if name == "count":
            continue
        for other in FORK:
            if other != name:
                assert fork(**{name: addr[other]}) == OVERLAP, (name, other)
    assert fork(status=addr["table_new"] + 4 * (5 * 9 + 7)) == OVERLAP and fork(status=addr["copies"] + 4 * 17) == OVERLAP
    assert fork(bytes=lb.lory_kv_fork_workspace_bytes(fork_shape()) - 1) == WORKSPACE


def copy_shape(**kw):
    d = dict(n=5, layers=2, pages=10, page=16, kv_heads=4, head_dim=64, dtype=B2)
    d.update(kw)
    return lb.LoryCopyShape(**d)


def copy(shape=None, **kw):
    a = dict(k_cache=F, v_cache=F + (1 << 30), copies=F + (1 << 32))
    a.update(kw)
    return lb.lib().lory_kv_copy(shape or copy_shape(), *a.values(), None)


@pytest.mark.parametrize("kw,rc", [(dict(n=-1), SHAPE), (dict(n=(1 << 20) + 1), SHAPE), (dict(layers=0), SHAPE), (dict(layers=32768), SHAPE),
                                   (dict(pages=0), SHAPE), (dict(page=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(head_dim=60), SHAPE),
                                   (dict(head_dim=264), SHAPE), (dict(pages=1 << 25), SHAPE), (dict(dtype=7), DTYPE),
                                   (dict(page=1 << 24, kv_heads=8, head_dim=256, pages=1, dtype=F4), SHAPE)])
def test_copy_shapes(kw, rc):
    assert copy(copy_shape(**kw)) == rc


def test_copy_arrays():
    assert lb.lib().lory_kv_copy(None, F, F, F, None) == NULL
    for name in ("k_cache", "v_cache", "copies"):
        assert copy(**{name: None}) == NULL
    assert copy(k_cache=F + 8) == copy(v_cache=F + 8) == copy(copies=F + (1 << 32) + 2) == ALIGN
    assert copy(v_cache=F + 16) == copy(copies=F + 64) == copy(v_cache=F + 2 * 10 * 16 * 4 * 64 * 2 - 16) == OVERLAP
    assert copy(copy_shape(n=0), copies=None) == lb.LORY_OK


def heads(data=F, token=512, head=64):
    return lb.LoryHeads(data, token, head)


def paged_shape(**kw):
    d = dict(rows=12, q_heads=8, kv_heads=4, head_dim=64, pages=20, page=16, width=8, dtype=B2, table_row=8, scale=0.125)
    d.update(kw)
    return lb.LoryPagedShape(**d)


def prefix(shape=None, groups=3, **kw):
    a = dict(q=heads(), k_cache=F, v_cache=F, table=F, lens=F, shared=F, out=heads(), lse=F, workspace=F, bytes=1 << 40)
    a.update(kw)
    return lb.lib().lory_prefix_attn(shape or paged_shape(), groups, *a.values(), None)


@pytest.mark.parametrize("kw,groups,rc", [(dict(), 5, SHAPE), (dict(), 0, SHAPE), (dict(), -1, SHAPE), (dict(), 13, SHAPE), (dict(rows=0), 1, SHAPE),
                                          (dict(rows=-1), 1, SHAPE), (dict(q_heads=6), 3, SHAPE), (dict(head_dim=60), 3, SHAPE),
                                          (dict(page=0), 3, SHAPE), (dict(table_row=7), 3, SHAPE), (dict(scale=0.0), 3, SHAPE),
                                          (dict(scale=float("nan")), 3, SHAPE), (dict(dtype=5), 3, DTYPE),
                                          (dict(rows=1 << 20, width=32720, table_row=32720, page=4), 1 << 10, SHAPE),
                                          (dict(rows=1 << 20, q_heads=65535, kv_heads=1), 1, SHAPE)])
def test_prefix_shapes(kw, groups, rc):
    assert prefix(paged_shape(**kw), groups) == rc
    assert lb.lib().lory_prefix_attn_workspace_bytes(paged_shape(**kw), groups, ctypes.byref(ctypes.c_size_t())) == rc


def test_prefix_arrays():
    for n in ("q", "k_cache", "v_cache", "table", "lens", "shared", "out", "workspace"):
        assert prefix(**{n: None}) == NULL, n
    for n in ("k_cache", "v_cache", "workspace"):
        assert prefix(**{n: F + 8}) == ALIGN, n
    for n in ("table", "lens", "shared", "lse"):
        assert prefix(**{n: F + 2}) == ALIGN, n
    assert prefix(q=heads(head=60)) == prefix(out=heads(token=100)) == ALIGN
    assert prefix(out=heads(head=0)) == OVERLAP
    assert prefix(bytes=lb.lory_prefix_attn_workspace_bytes(paged_shape(), 3) - 1) == WORKSPACE
    assert lb.lib().lory_prefix_attn(None, 1, heads(), F, F, F, F, F, heads(), F, F, 1, None) == NULL
    none = heads(data=None)
    assert prefix(paged_shape(rows=0), 0, q=none, out=none, table=None, lens=None, shared=None) == lb.LORY_OK


def test_binding_refuses_wrong_tensors():
    """Types, shapes and strides are checked before devices, so CPU tensors reach every check."""
    def bad(error, match, f, *args, **kw):
        with pytest.raises(error, match=match):
            f(*args, **kw)

    x, score = torch.zeros(6, 50), torch.zeros(2, 3)
    sel = lb.lory_beam_select
    bad(ValueError, "GPU", sel, x, score, 4)
    bad(ValueError, r"logits must be \[6, vocab\]", sel, x[:5], score, 4)
    bad(ValueError, "contiguous rows", sel, torch.zeros(6, 100)[:, ::2], score, 4)
    bad(TypeError, "unsupported dtype Half", sel, x.half(), score, 4)
    bad(ValueError, "score must be fp32", sel, x, score.double(), 4)
    bad(ValueError, "score must be fp32", sel, x, score.view(-1), 4)
    bad(ValueError, "token must be Int", sel, x, score, 4, token=torch.zeros(2, 4))
    bad(ValueError, r"score_out must be Float \[2, 4\]", sel, x, score, 4, score_out=torch.zeros(2, 5))
    bad(ValueError, "parent must be contiguous", sel, x, score, 4, parent=torch.zeros(4, 2, dtype=torch.int32).T)
    bad(ValueError, "k is too large", sel, x, score, 1 << 40)

    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    args = [i(3), i(5), i(3, 4), i(9), i(1), 16, 20, i(5), i(5, 4), i(1), i(3, 5), i(1)]
    bad(ValueError, "GPU", lb.lory_kv_fork, *args)
    for at, (wrong, match) in {0: (i(3).long(), "lens must be Int"), 2: (i(2, 4), "table must be int32"), 4: (i(2), "count must be"),
                               7: (i(4), "lens_new must be Int .5."), 8: (i(5, 3), "table_new must have the width"),
                               10: (i(2, 5), "copies must be int32"), 11: (i(2), "status must be")}.items():
        bad(ValueError, match, lb.lory_kv_fork, *args[:at], wrong, *args[at + 1:])

    k = torch.zeros(5, 2, 16, 64)
    bad(ValueError, "GPU", lb.lory_kv_copy, k, k, i(3, 4))
    bad(ValueError, "copies must be int32", lb.lory_kv_copy, k, k, i(4, 3))
    bad(ValueError, "copies must be int32", lb.lory_kv_copy, k, k, i(3, 4).long())
    bad(ValueError, "k_cache and v_cache must be", lb.lory_kv_copy, k, k[:4], i(3, 4))
    bad(ValueError, "k_cache and v_cache must be", lb.lory_kv_copy, k[0], k[0], i(3, 4))
    bad(TypeError, "v_cache must be Float", lb.lory_kv_copy, k, k.bfloat16(), i(3, 4))
    bad(ValueError, "k_cache must be contiguous", lb.lory_kv_copy, k[:, :, ::2], k[:, :, ::2], i(3, 4))

    q, table, lens = torch.zeros(6, 4, 64), i(6, 4), i(6)
    attn = lb.lory_prefix_attn
    bad(ValueError, "GPU", attn, q, k, k, table, lens, i(2))
    bad(ValueError, "6 rows, 4 groups", attn, q, k, k, table, lens, i(4))
    bad(ValueError, "6 rows, 0 groups", attn, q, k, k, table, lens, i(0))
    bad(ValueError, "shared must be Int", attn, q, k, k, table, lens, i(2).long())
    bad(ValueError, "lens must be Int .6.", attn, q, k, k, table, i(5), i(2))
    bad(ValueError, "lse must be fp32 .6, 4.", attn, q, k, k, table, lens, i(2), lse=torch.zeros(6, 2))
    bad(TypeError, "out must be Float", attn, q, k, k, table, lens, i(2), out=q.double())
