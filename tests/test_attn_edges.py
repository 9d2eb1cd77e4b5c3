"""The attention operators where a value, a layout or a step is out of the ordinary.  Plain implementations in 64 bits; bounds
as in test_attn_gpu.py."""
import os
import re

import numpy as np
import pytest
import torch

import test_attn_gpu as base
from paper_2405_03133_amd import autograd
from paper_2405_03133_amd import binding as lb
from test_attn_gpu import E32, T, attend, check_attention, freqs, gen, paged_case, rnd, within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


# Head counts that are no multiple of the heads of a load, and tokens on both sides of where one workgroup takes them all.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot,inter", [(2, 3, 1, 64, 64, False), (500, 3, 1, 64, 64, True), (16, 4, 4, 64, 32, False),
                                                  (300, 5, 2, 128, 128, False), (5, 9, 3, 80, 80, True), (41, 1, 1, 256, 0, False),
                                                  (1200, 8, 8, 8, 0, False), (33, 8, 4, 32, 32, False)])
def test_rope_gradient_without_eps(n, Hq, Hkv, D, rot, inter, dtype, monkeypatch):
    monkeypatch.setattr(base, "EPS", 0.0)
    base.test_rope_gradient(n, Hq, Hkv, D, rot, inter, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_at_any_address(dtype):
    """A gradient that autograd hands over as a contiguous view into a larger one, an element behind a multiple of 16 bytes."""
    t = T[dtype]
    g = gen(31)
    one = torch.ones(1, device="cuda", dtype=t)

    def grads(f, leaves, shift):
        leaves = [x.clone().requires_grad_() for x in leaves]
        loss = 0.0
        for y, c in zip(f(*leaves), factors):
            loss = loss + (torch.cat([one] * shift + [y.reshape(-1)]) * torch.cat([one] * shift + [c])).sum()
        return torch.autograd.grad(loss, leaves)

    n, Hq, Hkv, D = 9, 3, 1, 64
    factors = [rnd(g, n * h * D, dtype=t) for h in (Hq, Hkv)]
    pos, freq = torch.arange(n, device="cuda", dtype=torch.int32), freqs(D)
    leaves = [rnd(g, n, Hq, D, dtype=t), rnd(g, n, Hkv, D, dtype=t), 1 + rnd(g, D, dtype=t) / 4, 1 + rnd(g, D, dtype=t) / 4]
    rope = lambda q, k, wq, wk: autograd.qk_rope(q, k, pos, freq, wq, wk)
    for a, b in zip(grads(rope, leaves, 0), grads(rope, leaves, 1)):
        assert torch.equal(a, b)
    B, L, seg, d, d_ff, E = 1, 128, 64, 128, 256, 4
    factors = [rnd(g, B * L * d, dtype=t)]
    leaves = [rnd(g, B, L, d, dtype=t), rnd(g, d, E, dtype=t) / 8] + [rnd(g, E, *s, dtype=t) / 8 for s in ((d, d_ff), (d, d_ff), (d_ff, d))]
    layer = lambda x, R, Wg, Wu, Wd: [autograd.lory_layer(x, R, Wg, Wu, Wd, seg)]
    for a, b in zip(grads(layer, leaves, 0), grads(layer, leaves, 1)):
        assert torch.equal(a, b)


def test_generation_snippet_of_the_readme_with_a_row_that_has_ended():
    """A step's tokens are packed, and a row that has ended has none: the rows behind it still attend with their own queries."""
    text = open(os.path.join(ROOT, "README.md")).read()
    code = re.search(r"^Generation:.*?```python\n(.*?)```", text, re.S | re.M).group(1)
    B, W, page, F, Hq, Hkv, D = 5, 8, 16, 60, 4, 2, 64
    g = gen(40)
    i32 = lambda a: torch.tensor(np.asarray(a).tolist(), dtype=torch.int32, device="cuda")
    held, add = [40, 17, 64, 5, 99], [1, -1, 1, -1, 1]
    blocks = [-(-n // page) for n in held]
    pages = np.random.RandomState(1).permutation(F)
    table, at = np.full((B, W), -1), 0
    for b, m in enumerate(blocks):
        table[b, :m] = pages[at:at + m]
        at += m
    free = np.full(F, -1)
    free[:F - at] = pages[at:]
    k_cache, v_cache = rnd(g, F, Hkv, page, D), rnd(g, F, Hkv, page, D)
    old = table.copy()
    qkv = rnd(g, B, (Hq + 2 * Hkv) * D)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    s = dict(torch=torch, lb=lb, lens=i32(held), add=i32(add), table=i32(table), free=i32(free), count=i32([F - at]), page=page,
             lens_new=i32([0] * B), cu=i32([0] * (B + 1)), positions=i32([0] * B), slots=torch.zeros(B, dtype=torch.int64, device="cuda"),
             count_new=i32([0]), status=i32([0]), q=q, k=k, v=v, freq=freqs(D), wq=1 + rnd(g, D) / 4, wk=1 + rnd(g, D) / 4,
             k_cache=k_cache, v_cache=v_cache)
    exec(code, s)
    assert s["status"].item() == 0
    live = [0, 2, 4]
    # the packed token i is that of the i-th live row: its query over that row's cache, the new key and value among them
    pos = i32([held[b] for b in live])
    yq, yk = lb.lory_qk_rope(q[:3], k[:3], pos, s["freq"], wq=s["wq"], wk=s["wk"])
    assert torch.equal(s["q"][:3], yq)
    for i, b in enumerate(live):
        row, n = s["table"][b], held[b] + 1
        assert row[:blocks[b]].tolist() == old[b, :blocks[b]].tolist()
        slot = int(row[held[b] // page]) * page + held[b] % page
        assert torch.equal(k_cache[slot // page, :, slot % page], yk[i]) and torch.equal(v_cache[slot // page, :, slot % page], v[i])
        lse = torch.empty(1, Hq, device="cuda")
        lb.lory_paged_attn(yq[i:i + 1], k_cache, v_cache, row[None], i32([n]), lse=lse)
        check_attention(f"row {b}", s["out"][i:i + 1], lse, yq[i:i + 1], k_cache, v_cache, row[None], i32([n]))
    assert (s["out"][3:] == 0).all()   # places without a token


def test_generation_snippet_of_the_readme_in_a_graph():
    """Steps in which rows end at random, captured once and replayed with the program's own work in between: every replay against
    the same step run eagerly, and every live row against 64 bits with its own query."""
    text = open(os.path.join(ROOT, "README.md")).read()
    code = compile(re.search(r"^Generation:.*?```python\n(.*?)```", text, re.S | re.M).group(1), "README.md", "exec")
    B, W, page, F, Hq, Hkv, D = 6, 4, 8, 40, 4, 2, 64
    g, rs = gen(41), np.random.RandomState(41)
    i32 = lambda a: torch.tensor(np.asarray(a).tolist(), dtype=torch.int32, device="cuda")
    wq, wk = 1 + rnd(g, D) / 4, 1 + rnd(g, D) / 4

    def fresh():
        qkv = torch.zeros(B, (Hq + 2 * Hkv) * D, device="cuda")
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
        kc, vc = (torch.zeros(F, Hkv, page, D, device="cuda") for _ in range(2))
        return dict(torch=torch, lb=lb, lens=i32([0] * B), add=i32([0] * B), table=i32(np.full((B, W), -1)), free=i32(range(F)), count=i32([F]),
                    page=page, lens_new=i32([0] * B), cu=i32([0] * (B + 1)), positions=i32([0] * B),
                    slots=torch.zeros(B, dtype=torch.int64, device="cuda"), count_new=i32([0]), status=i32([0]), q=q, k=k, v=v, freq=freqs(D),
                    wq=wq, wk=wk, k_cache=kc, v_cache=vc), qkv

    def step(s, q):
        s["q"] = q
        exec(code, s)
        s["lens"].copy_(s["lens_new"])
        s["count"].copy_(s["count_new"])

    (eager, eager_qkv), (captured, captured_qkv) = fresh(), fresh()
    eager_q, captured_q = eager["q"], captured["q"]
    step(fresh()[0], eager_q.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured, captured_q)
    ended = 0
    for i in range(20):
        add = np.where(rs.rand(B) < 0.2, -1, np.where(rs.rand(B) < 0.2, 0, 1))
        qkv = rnd(g, B, (Hq + 2 * Hkv) * D)
        for s, x in ((eager, eager_qkv), (captured, captured_qkv)):
            s["add"].copy_(i32(add))
            x.copy_(qkv)
        step(eager, eager_q)
        graph.replay()
        junk = torch.randn(1000, 1000, device="cuda")
        (junk @ junk).sum().item()
        for n in ("lens", "count", "table", "free", "cu", "positions", "slots", "status", "k_cache", "v_cache", "q", "out"):
            assert torch.equal(captured[n], eager[n]), (i, n)
        assert eager["status"].item() == 0
        lens, live = eager["lens"].tolist(), [b for b in range(B) if add[b] > 0]
        ended += (add < 0).sum()
        for t, b in enumerate(live):
            y, row, n = eager["q"][t:t + 1], eager["table"][b:b + 1], i32([lens[b]])
            lse = torch.empty(1, Hq, device="cuda")
            lb.lory_paged_attn(y, eager["k_cache"], eager["v_cache"], row, n, lse=lse)
            check_attention(f"step {i} row {b}", eager["out"][t:t + 1], lse, y, eager["k_cache"], eager["v_cache"], row, n)
    assert ended > 5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,Hq,Hkv,D,page", [([1, 37, 200], 2, 1, 64, 16), ([1, 130, 9], 17, 1, 40, 8), ([5000, 1, 64], 8, 2, 128, 16),
                                                ([1, 300], 4, 2, 256, 16), ([333, 4000], 20, 4, 80, 24)])
def test_attention_of_infinite_values(lens, Hq, Hkv, D, page, dtype):
    """A value of a token that counts may be infinite: so is its dim of every query of the head, NaN where both signs meet;
    all other dims are what they are without it."""
    q, k, v, table, dlens = paged_case(sum(lens), lens, Hq, Hkv, D, page, dtype, sigma=0.5)
    plain = attend((q, k, v, table, dlens))
    inf = float("inf")
    v = v.clone()
    for b, n in enumerate(lens):
        for t, d, x in ((0, 0, inf), (n - 1, D - 1, -inf), (n // 2, D // 2, inf), (n // 3, 5, inf), (n - 1, 5, -inf), (n // 4, 6, float("nan"))):
            if n > 1 or d != 5:
                v[int(table[b, t // page]), Hkv - 1, t % page, d] = x
    out, lse = attend((q, k, v, table, dlens))
    check_attention("infinite values", out, lse, q, k, v, table, dlens)
    last = out[:, -(Hq // Hkv):]
    for b, n in enumerate(lens):
        assert (last[b, :, 0] == inf).all() and (last[b, :, D - 1] == -inf).all() and (last[b, :, D // 2] == inf).all()
        assert torch.isnan(last[b, :, 6]).all() and (n == 1 or torch.isnan(last[b, :, 5]).all())
    odd = torch.zeros(D, dtype=torch.bool, device="cuda")
    odd[[0, 5, 6, D // 2, D - 1]] = True
    assert torch.equal(lse, plain[1]) and torch.equal(out[..., ~odd], plain[0][..., ~odd])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("scale", [0.5, 0.7, 1.0])
@pytest.mark.parametrize("lens", [[200, 1, 65], [9000, 200, 3]])
def test_attention_scores_at_the_ends_of_their_range(lens, scale, sign, dtype):
    """Head 0's scores are all scale times the type's lowest (or largest) value; head 1's are that and, every third, 0.  Any
    score that fp32 holds counts as it is: equal ones weigh alike, and beside a 0 the lowest ones nothing."""
    t, D, page = T[dtype], 64, 16
    q, k, v, table, dlens = paged_case(7 + len(lens), lens, 2, 2, D, page, dtype, sigma=1.0)
    end = sign * torch.finfo(t).max
    q.zero_()
    q[..., 0] = 1
    for b, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        p = table[b].long()[i // page]
        k[p, :, i % page] = 0
        k[p, 0, i % page, 0] = end
        k[p, 1, i % page, 0] = torch.where(i % 3 == 0, 0.0, end).to(t)
    out, lse = attend((q, k, v, table, dlens), scale=scale)
    for b, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        V = v[table[b].long()[i // page], :, i % page].double()
        for h in range(2):
            keep = torch.ones_like(i, dtype=torch.bool) if h == 0 else i % 3 == 0 if sign < 0 else (i % 3 != 0) | (n == 1)
            ref = V[keep, h].mean(0)
            # as the plain means of test_attention_extreme_scores; sums of equal weights in chains of at most n / 16 + 64
            within(f"{n} scores, head {h}", out[b, h], ref, (2.0 ** -16 + (8 + 2 * (n / 16 + 64)) * E32) * V[keep, h].abs().mean(0), t)
            top = 0.0 if h == 1 and (sign < 0 or n == 1) else scale * end
            want = top + float(np.log(keep.sum().item()))
            assert abs(lse[b, h].item() - want) <= (4 + n / 16 + 64 + 8 * abs(want)) * E32, (n, h, lse[b, h].item(), want)


def test_writes_are_seen_by_autograd():
    """Tensors that a call writes into count as changed: a graph that kept one of them raises instead of using the new values."""
    g = gen(50)
    n, H, D, page = 4, 2, 64, 16
    x, pos, freq, w = rnd(g, n, H, D), torch.arange(n, device="cuda", dtype=torch.int32), freqs(64), torch.ones(D, device="cuda")
    kc, vc = torch.zeros(2, H, page, D, device="cuda"), torch.zeros(2, H, page, D, device="cuda")
    table, slots = torch.zeros(n, 1, dtype=torch.int32, device="cuda"), torch.arange(n, device="cuda")
    out = [torch.empty_like(x) for _ in range(2)]
    dw, lse = [torch.empty(D, device="cuda") for _ in range(2)], torch.empty(n, H, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    plan = [i32(3), i32(1), i32(0, 0)[None].clone(), i32(1, 2), i32(2), 16, i32(0), i32(0, 0), i32(0), torch.zeros(1, dtype=torch.int64, device="cuda"), i32(0), i32(0)]
    calls = [(lambda: lb.lory_qk_rope(x, x, pos, freq, q_out=out[0], k_out=out[1]), out, [x, pos, freq]),
             (lambda: lb.lory_qk_rope_cache(x, x, x, pos, freq, kc, vc, slots, q_out=out[0], wq=w, wk=w), [kc, vc, out[0]], [x, slots, w]),
             (lambda: lb.lory_qk_rope_bwd(x, x, x, x, pos, freq, w, w, dq=out[0], dk=out[1], dwq=dw[0], dwk=dw[1]), out + dw, [x, w]),
             (lambda: lb.lory_paged_attn(x, kc, vc, table, pos, out=out[0], lse=lse), [out[0], lse], [x, kc, vc, table, pos]),
             (lambda: lb.lory_kv_plan(*plan), plan[2:4] + plan[6:], [plan[0], plan[1], plan[4]])]
    for i, (call, written, read) in enumerate(calls):
        before = [t._version for t in written], [t._version for t in read]
        call()
        assert all(t._version > v for t, v in zip(written, before[0])), i
        assert [t._version for t in read] == before[1], i
    leaf = x.clone().requires_grad_()
    h = leaf * 1.0
    y = (h * h).sum()   # keeps h
    lb.lory_qk_rope(h.detach(), x, pos, freq, q_out=h.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():
        a = torch.empty_like(x)
    lb.lory_qk_rope(x, x, pos, freq, q_out=a)   # a tensor without a version
    assert torch.equal(a, lb.lory_qk_rope(x, x, pos, freq)[0])
