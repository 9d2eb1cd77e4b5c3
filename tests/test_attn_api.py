"""Argument checks and index arithmetic of the attention operators.  No GPU: every call returns from validation, and the
arithmetic that keeps accesses in bounds is compiled for the host."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2405_03133_amd import binding as lb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = 0x7F0000001000   # aligned, never dereferenced on these paths
B2, F4 = lb.LORY_BF16, lb.LORY_F32


def heads(data=F, token=512, head=64):
    return lb.LoryHeads(data, token, head)


def rope_shape(**kw):
    d = dict(tokens=10, q_heads=8, kv_heads=8, head_dim=64, rot_dim=64, interleaved=0, dtype=B2, eps=1e-6)
    d.update(kw)
    return lb.LoryRopeShape(**d)


def rope(shape=None, **kw):
    a = dict(q=heads(), k=heads(), pos=F, freq=F, wq=F, wk=F, q_out=heads(), k_out=heads())
    a.update(kw)
    return lb.lib().lory_qk_rope(shape or rope_shape(), *a.values(), None)


def store(shape=None, **kw):
    a = dict(q=heads(), k=heads(), v=heads(), pos=F, freq=F, wq=F, wk=F, q_out=heads(), k_cache=F, v_cache=F, pages=4,
             page=16, slots=F)
    a.update(kw)
    return lb.lib().lory_qk_rope_cache(shape or rope_shape(), *a.values(), None)


def bwd(shape=None, **kw):
    shape = shape or rope_shape()
    a = dict(q=heads(), k=heads(), dq_out=heads(), dk_out=heads(), pos=F, freq=F, wq=F, wk=F, dq=heads(), dk=heads(), dwq=F,
             dwk=F, workspace=F, bytes=lb.lory_qk_rope_workspace_bytes(rope_shape()))
    a.update(kw)
    return lb.lib().lory_qk_rope_bwd(shape, *a.values(), None)


BAD_ROPE = [(dict(tokens=-1), lb.LORY_ERR_SHAPE), (dict(tokens=(1 << 25) + 1), lb.LORY_ERR_SHAPE),
            (dict(q_heads=0), lb.LORY_ERR_SHAPE), (dict(kv_heads=0), lb.LORY_ERR_SHAPE), (dict(q_heads=65536), lb.LORY_ERR_SHAPE),
            (dict(head_dim=0), lb.LORY_ERR_SHAPE), (dict(head_dim=68), lb.LORY_ERR_SHAPE), (dict(head_dim=264), lb.LORY_ERR_SHAPE),
            (dict(rot_dim=8), lb.LORY_ERR_SHAPE), (dict(rot_dim=80), lb.LORY_ERR_SHAPE), (dict(rot_dim=-16), lb.LORY_ERR_SHAPE),
            (dict(interleaved=2), lb.LORY_ERR_SHAPE), (dict(eps=-1.0), lb.LORY_ERR_SHAPE), (dict(eps=float("nan")), lb.LORY_ERR_SHAPE),
            (dict(eps=float("inf")), lb.LORY_ERR_SHAPE), (dict(dtype=2), lb.LORY_ERR_DTYPE)]


@pytest.mark.parametrize("call", [rope, store, bwd])
@pytest.mark.parametrize("kw,rc", BAD_ROPE)
def test_rope_shapes(call, kw, rc):
    assert call(rope_shape(**kw)) == rc


@pytest.mark.parametrize("call,names", [(rope, ["q", "k", "q_out", "k_out"]), (store, ["q", "k", "v", "q_out"]),
                                        (bwd, ["q", "k", "dq_out", "dk_out", "dq", "dk"])])
def test_rope_heads(call, names):
    for n in names:
        assert call(**{n: None}) == lb.LORY_ERR_NULL, n
        assert call(**{n: heads(data=None)}) == lb.LORY_ERR_NULL, n
        assert call(**{n: heads(data=F + 8)}) == lb.LORY_ERR_ALIGN, n
        assert call(**{n: heads(token=516)}) == lb.LORY_ERR_ALIGN, n
        assert call(**{n: heads(head=68)}) == lb.LORY_ERR_ALIGN, n
        assert call(**{n: heads(token=-512)}) == lb.LORY_ERR_SHAPE, n
        out = n in ("q_out", "k_out", "dq", "dk")
        if out:
            assert call(**{n: heads(token=504)}) == lb.LORY_ERR_OVERLAP, n      # the last head reaches into the next token
            assert call(**{n: heads(head=56)}) == lb.LORY_ERR_OVERLAP, n
            assert call(**{n: heads(token=64, head=632)}) == lb.LORY_ERR_OVERLAP, n   # heads outside, ten tokens of 64 in each
            assert call(**{n: heads(token=0)}) == lb.LORY_ERR_OVERLAP, n


@pytest.mark.parametrize("call,names", [(rope, ["pos", "freq"]), (store, ["pos", "freq", "k_cache", "v_cache", "slots"]),
                                        (bwd, ["pos", "freq", "dwq", "dwk", "workspace"])])
def test_rope_arrays(call, names):
    for n in names:
        assert call(**{n: None}) == lb.LORY_ERR_NULL, n
        assert call(**{n: F + 2}) == lb.LORY_ERR_ALIGN, n
    assert call(wq=None) == lb.LORY_ERR_NULL
    assert call(wk=None) == lb.LORY_ERR_NULL
    assert call(wq=F + 8) == lb.LORY_ERR_ALIGN


def test_rope_other_refusals():
    assert store(pages=0) == store(page=0) == store(page=-1) == lb.LORY_ERR_SHAPE
    assert store(pages=1 << 20, page=1 << 11) == lb.LORY_ERR_SHAPE            # 2^31 rows of one head
    assert store(pages=1 << 14, page=1 << 14) == lb.LORY_ERR_SHAPE            # with 8 heads
    n = lb.lory_qk_rope_workspace_bytes(rope_shape())
    assert n > 0 and bwd(bytes=n - 1) == lb.LORY_ERR_WORKSPACE
    assert lb.lib().lory_qk_rope_workspace_bytes(rope_shape(), None) == lb.LORY_ERR_NULL
    assert lb.lib().lory_qk_rope_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == lb.LORY_ERR_NULL


def test_nothing_to_do_needs_no_memory():
    none = heads(data=None)
    s = rope_shape(tokens=0)
    assert rope(s, q=none, k=none, pos=None, q_out=none, k_out=none) == lb.LORY_OK
    assert store(s, q=none, k=none, v=none, pos=None, q_out=none, slots=None) == lb.LORY_OK
    assert bwd(s, q=none, k=none, dq_out=none, dk_out=none, pos=None, dq=none, dk=none, wq=None, wk=None, dwq=None, dwk=None,
               workspace=None, bytes=0) == lb.LORY_OK
    assert lb.lory_qk_rope_workspace_bytes(s) == 0
    assert paged(paged_shape(rows=0), q=none, out=none, table=None, lens=None) == lb.LORY_OK


# ---------------------------------------------------------------- plan

def plan_shape(**kw):
    d = dict(rows=4, width=8, page=16, free_size=64, room=32, table_row=8)
    d.update(kw)
    return lb.LoryPlanShape(**d)


ARRAYS = ("lens", "add", "table", "free", "count", "lens_new", "cu", "positions", "slots", "count_new", "status")


def plan(shape=None, **kw):
    a = {n: F + 0x1000 * i for i, n in enumerate(ARRAYS)}
    a.update(kw)
    return lb.lib().lory_kv_plan(shape or plan_shape(), *a.values(), None)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=(1 << 20) + 1), dict(room=-1), dict(width=0), dict(page=0),
                                dict(free_size=0), dict(table_row=7), dict(width=1 << 16, table_row=1 << 16, page=1 << 15)])
def test_plan_shapes(kw):
    assert plan(plan_shape(**kw)) == lb.LORY_ERR_SHAPE


def test_plan_arrays():
    assert lb.lib().lory_kv_plan(None, *[F] * 11, None) == lb.LORY_ERR_NULL
    for n in ARRAYS:
        assert plan(**{n: None}) == lb.LORY_ERR_NULL, n
        assert plan(**{n: F + 0x100000 + 2}) == lb.LORY_ERR_ALIGN, n
    assert plan(slots=F + 0x100000 + 4) == lb.LORY_ERR_ALIGN
    addr = {n: F + 0x1000 * i for i, n in enumerate(ARRAYS)}
    for n in ARRAYS[2:]:
        if n == "count":
            continue
        for other in ARRAYS:
            if other != n:
                assert plan(**{n: addr[other]}) == lb.LORY_ERR_OVERLAP, (n, other)
    # the last place of the table's last row
    assert plan(plan_shape(table_row=100), cu=addr["table"] + 4 * (3 * 100 + 7)) == lb.LORY_ERR_OVERLAP


# ---------------------------------------------------------------- attention

def paged_shape(**kw):
    d = dict(rows=10, q_heads=8, kv_heads=4, head_dim=64, pages=20, page=16, width=8, dtype=B2, table_row=8, scale=0.125)
    d.update(kw)
    return lb.LoryPagedShape(**d)


def paged(shape=None, **kw):
    shape = shape or paged_shape()
    a = dict(q=heads(), k_cache=F, v_cache=F, table=F, lens=F, out=heads(), lse=F, workspace=F, bytes=1 << 30)
    a.update(kw)
    return lb.lib().lory_paged_attn(shape, *a.values(), None)


@pytest.mark.parametrize("kw,rc", [(dict(rows=-1), 2), (dict(rows=(1 << 20) + 1), 2), (dict(q_heads=6), 2), (dict(kv_heads=0), 2),
                                   (dict(head_dim=60), 2), (dict(head_dim=512), 2), (dict(pages=0), 2), (dict(page=0), 2),
                                   (dict(width=0), 2), (dict(table_row=7), 2), (dict(scale=0.0), 2), (dict(scale=-1.0), 2),
                                   (dict(scale=float("nan")), 2), (dict(scale=float("inf")), 2), (dict(dtype=5), 3),
                                   (dict(width=1 << 20, table_row=1 << 20, page=1025), 2), (dict(pages=1 << 25), 2),
                                   (dict(rows=1 << 20, width=1 << 17, table_row=1 << 17), 2)])
def test_paged_shapes(kw, rc):
    assert paged(paged_shape(**kw)) == rc


def test_paged_arrays():
    for n in ("q", "k_cache", "v_cache", "table", "lens", "out", "workspace"):
        assert paged(**{n: None}) == lb.LORY_ERR_NULL, n
    for n in ("k_cache", "v_cache", "workspace"):
        assert paged(**{n: F + 8}) == lb.LORY_ERR_ALIGN, n
    for n in ("table", "lens", "lse"):
        assert paged(**{n: F + 2}) == lb.LORY_ERR_ALIGN, n
    assert paged(q=heads(head=60)) == paged(out=heads(token=100)) == lb.LORY_ERR_ALIGN
    assert paged(out=heads(head=0)) == paged(out=heads(token=448 + 56)) == lb.LORY_ERR_OVERLAP
    n = lb.lory_paged_attn_workspace_bytes(paged_shape())
    assert paged(bytes=n - 1) == lb.LORY_ERR_WORKSPACE
    assert lb.lib().lory_paged_attn(None, heads(), F, F, F, F, heads(), F, F, n, None) == lb.LORY_ERR_NULL


def test_status_of_overlaps_has_a_text():
    assert len({lb.status_string(i) for i in range(8)}) == 8 and lb.status_string(lb.LORY_ERR_OVERLAP) != "unknown status"


# ---------------------------------------------------------------- the binding's own checks

def test_binding_refuses_wrong_tensors():
    """Types, shapes and strides are checked before devices, so CPU tensors reach every check."""
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    pos, freq, w = torch.zeros(3, dtype=torch.int32), torch.zeros(32, dtype=torch.float64), torch.ones(64)

    def refused(error, match, f, *args, **kw):
        with pytest.raises(error, match=match):
            f(*args, **kw)

    rope, bad = lb.lory_qk_rope, refused
    bad(ValueError, "GPU", rope, q, k, pos, freq)
    bad(ValueError, "last dimension of q .* contiguous", rope, torch.zeros(3, 4, 128)[..., ::2], k, pos, freq)
    bad(TypeError, "k must be Float", rope, q, k.double(), pos, freq)
    bad(TypeError, "unsupported dtype Half", rope, q.half(), k.half(), pos, freq)
    bad(ValueError, r"k must be \[3, 2, 64\]", rope, q, k[..., :32], pos, freq)
    bad(ValueError, "q and k must be", rope, q[0], k, pos, freq)
    bad(ValueError, "pos must be Int", rope, q, k, pos.long(), freq)
    bad(ValueError, "pos must be Int .3.", rope, q, k, pos[:2], freq)
    bad(ValueError, "pos must be contiguous", rope, q, k, torch.zeros(6, dtype=torch.int32)[::2], freq)
    bad(ValueError, "freq must be Double", rope, q, k, pos, freq.float())
    bad(TypeError, "wq must be Float", rope, q, k, pos, freq, wq=w.bfloat16(), wk=w)
    bad(ValueError, "wk must be Float .64.", rope, q, k, pos, freq, wq=w, wk=w[:32])
    bad(ValueError, "q_out must be", rope, q, k, pos, freq, q_out=k)
    bad(TypeError, "k_out must be", rope, q, k, pos, freq, k_out=k.bfloat16())
    bad(TypeError, "q must be a tensor", rope, None, k, pos, freq)
    bad(TypeError, "number", rope, q, k, pos, freq, eps="x")
    bad(ValueError, "GPU", rope, torch.zeros(3, 4, 64, device="meta"), k, pos, freq)

    cache, slots = torch.zeros(5, 2, 16, 64), torch.zeros(3, dtype=torch.int64)
    store = lambda v=k, kc=cache, vc=cache, s=slots: lb.lory_qk_rope_cache(q, k, v, pos, freq, kc, vc, s)
    bad(ValueError, "GPU", store)
    bad(ValueError, "v must be", store, v=q)
    bad(ValueError, "k_cache and v_cache must be", store, kc=cache[:, :1])
    bad(ValueError, "k_cache and v_cache must be", store, vc=cache[:4])
    bad(TypeError, "v_cache must be Float", store, vc=cache.bfloat16())
    bad(ValueError, "k_cache must be contiguous", store, kc=torch.zeros(5, 2, 32, 64)[:, :, ::2])
    bad(ValueError, "slots must be Long", store, s=slots.int())

    grad = lb.lory_qk_rope_bwd
    bad(ValueError, "GPU", grad, q, k, q, k, pos, freq, w, w)
    bad(ValueError, "dk_out must be", grad, q, k, q, q, pos, freq)
    bad(ValueError, "dwq and dwk need", grad, q, k, q, k, pos, freq, dwq=w)
    bad(ValueError, "dwk must be Float .64.", grad, q, k, q, k, pos, freq, w, w, dwk=w[:1])

    table = torch.zeros(3, 4, dtype=torch.int32)
    attn = lb.lory_paged_attn
    bad(ValueError, "GPU", attn, q, cache, cache, table, pos)
    bad(ValueError, "k_cache and v_cache must be", attn, q, cache[..., :32], cache, table, pos)
    bad(TypeError, "k_cache must be Float", attn, q, cache.bfloat16(), cache, table, pos)
    bad(ValueError, "table must be int32", attn, q, cache, cache, table.long(), pos)
    bad(ValueError, "table must be int32", attn, q, cache, cache, table[:2], pos)
    bad(ValueError, "table must be int32", attn, q, cache, cache, torch.zeros(4, 3, dtype=torch.int32).T, pos)
    bad(ValueError, "lens must be Int .3.", attn, q, cache, cache, table, pos[:1])
    bad(ValueError, "lse must be fp32 .3, 4.", attn, q, cache, cache, table, pos, lse=torch.zeros(3, 2))
    bad(TypeError, "out must be Float", attn, q, cache, cache, table, pos, out=q.double())

    i = lambda n: torch.zeros(n, dtype=torch.int32)
    args = [i(3), i(3), table, i(9), i(1), 16, i(3), i(4), i(8), torch.zeros(8, dtype=torch.int64), i(1), i(1)]
    bad(ValueError, "GPU", lb.lory_kv_plan, *args)
    for at, (wrong, match) in {1: (i(2), "add must be"), 4: (i(2), "count must be"), 7: (i(3), "cu must be Int .4."),
                               9: (i(8), "slots must be Long"), 10: (i(1).long(), "count_new must be Int")}.items():
        bad(ValueError, match, lb.lory_kv_plan, *args[:at], wrong, *args[at + 1:])
    bad(ValueError, "page is too large", lb.lory_kv_plan, *args[:5], 1 << 40, *args[6:])


# ---------------------------------------------------------------- index arithmetic

HOST = r"""
#include <stdio.h>
#include "paged_index.h"
using namespace lory::paged;
int main()
{
    long bad = 0;
    unsigned rng = 1;
    auto rnd = [&]() { return rng = rng * 1664525u + 1013904223u; };
    // quotients, at the multiples of the page and beside them, up to the largest token
    for (int i = 0; i < 4000; ++i) {
        const int page = i < 1000 ? i + 1 : i < 1032 ? 1 << (i - 1000) & 0x7fffffff : (int)(rnd() >> (1 + rnd() % 30)) + 1;
        if (page <= 0) continue;
        const Divider d = divider(page);
        for (int j = 0; j < 300; ++j) {
            const unsigned t0 = j == 0 ? 0x7fffffffu : j == 1 ? 0 : rnd() >> (1 + j % 24), m = t0 / page * page;
            const unsigned ts[3] = {t0, m, m ? m - 1 : 0};
            for (unsigned t : ts) bad += quotient(d, t) != t / page;
        }
    }
    // rows: inside the cache for every page number there is, -1 for every other
    for (int i = 0; i < 200000; ++i) {
        const int pages = 1 + rnd() % 50, heads = 1 + rnd() % 9, page = 1 + rnd() % 40, head = rnd() % heads;
        const unsigned t = rnd() >> 1;
        const int at = i % 3 ? (int)(rnd() % (pages + 4)) - 2 : (int)rnd();
        const Divider d = divider(page);
        const int row = cache_row(d, t, at, pages, heads, head);
        if (at < 0 || at >= pages) bad += row != -1;
        else bad += row != (at * heads + head) * page + (int)(t % page) || row < 0 || row >= pages * heads * page;
    }
    // ranges: in order, nothing left out, and every unit found in its own
    for (int i = 0; i < 300; ++i) {
        const int groups = i % 2 ? 512 : 1 + rnd() % 700;
        const long U = 1 + (i < 100 ? i : rnd() % 20000);
        bad += range_begin(0, U, groups) != 0 || range_begin(groups, U, groups) != U;
        for (int w = 0; w < groups; ++w) {
            const long a = range_begin(w, U, groups), b = range_begin(w + 1, U, groups);
            bad += b < a;
            for (long u = a; u < b; ++u) bad += owner(u, U, groups) != w;
        }
    }
    const long huge = (1l << 47);
    for (int w = 0; w < 512; ++w) {
        const long a = range_begin(w, huge + 77, 512);
        bad += owner(a, huge + 77, 512) != w || (w && owner(a - 1, huge + 77, 512) != w - 1);
    }
    printf("bad %ld\n", bad);
    return bad != 0;
}
"""


def test_index_arithmetic_on_the_host(tmp_path):
    src, exe = tmp_path / "t.cpp", str(tmp_path / "t")
    src.write_text(HOST)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I",
                    os.path.join(ROOT, "paper_2405_03133_amd", "csrc"), "-o", exe, str(src)], check=True)
    out = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "bad 0", out.stdout[-2000:]
