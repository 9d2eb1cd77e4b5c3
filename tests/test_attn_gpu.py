"""The attention operators against plain implementations in 64 bits.

Bounds are counted, not measured: u(T) = finfo(T).eps / 2 for the last rounding of a value, and multiples of 2^-24 of the sizes of
the terms for what is done in fp32 (the multiples are at each check)."""
import math

import numpy as np
import pytest
import torch

from paper_2405_03133_amd import binding as lb

pytestmark = pytest.mark.gpu

T = {"bf16": torch.bfloat16, "f32": torch.float32}
E32 = 2.0 ** -24
EPS = 1e-6


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rnd(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def within(label, got, ref, bound, dtype=None):
    """|got - ref| <= bound + the rounding to dtype, everywhere; NaN and infinities where the reference has them."""
    if dtype is not None:
        bound = bound + torch.finfo(dtype).eps / 2 * ref.abs()
    got = got.double()
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    err = torch.where(same, torch.zeros_like(ref), (got - ref).abs() - bound)
    worst = err.max().item() if err.numel() else 0.0
    print(f"[attn] {label}: worst excess {worst:.2e}", flush=True)
    assert not torch.isnan(err).any() and worst <= 0.0, (label, worst, (err > 0).sum().item())


# ---------------------------------------------------------------- norm and rotation

def freqs(rot):
    return torch.from_numpy(10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))).cuda()


def halves(x, rot, inter):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])


def join(x, a, b, rot, inter):
    y = x.clone()
    if inter:
        y[..., 0:rot:2], y[..., 1:rot:2] = a, b
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = a, b
    return y


def turned(x, pos, freq, inter, sign=1.0, magnitude=False):
    rot = 2 * freq.numel()
    t = (pos.double()[:, None] * freq)[:, None, :]
    c, s = t.cos(), sign * t.sin()
    a, b = halves(x, rot, inter)
    if magnitude:
        a, b, c, s = a.abs(), b.abs(), c.abs(), s.abs()
        # the angle: four roundings of fp64 between the operator and the reference
        far = 4 * 2.0 ** -53 * t.abs() / ROPE * (a + b)
        return join(x.abs(), a * c + b * s + far, b * c + a * s + far, rot, inter)
    return join(x, a * c - b * s, b * c + a * s, rot, inter)


def rope_ref(x, w, pos, freq, inter):
    """(y, size of its terms) in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    return turned(x, pos, freq, inter), turned(x, pos, freq, inter, magnitude=True)


# Terms of y: x, r, w, cos or sin.  r carries the sum of squares (at most 8 additions in a lane and 6 over lanes, halved by
# the root), division and root (4); cos and sin are good to 2 (reduced angle, function); 3 products, 1 addition.
ROPE = 24 * E32

SHAPES = [(1, 1, 1, 8, 0), (1, 16, 16, 64, 64), (3, 5, 5, 64, 32), (7, 12, 4, 80, 32), (7, 4, 4, 80, 80), (257, 3, 1, 96, 96),
          (33, 9, 3, 128, 128), (64, 16, 2, 128, 32), (5, 70, 10, 128, 128), (5000, 2, 1, 64, 64), (2, 8, 8, 256, 256),
          (9, 6, 2, 200, 16), (4, 7, 1, 32, 32), (11, 3, 3, 16, 16), (6, 2, 2, 40, 32), (3, 1, 1, 248, 240)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot", SHAPES)
def test_rope(n, Hq, Hkv, D, rot, inter, dtype):
    g = gen(n + D)
    t = T[dtype]
    q, k = rnd(g, n, Hq, D, dtype=t), 3 * rnd(g, n, Hkv, D, dtype=t)
    wq, wk = (1 + 0.3 * rnd(g, D)).to(t), (1 + 0.3 * rnd(g, D)).to(t)
    pos = torch.randint(-50, 5000, (n,), device="cuda", dtype=torch.int32)
    freq = freqs(rot)
    yq, yk = lb.lory_qk_rope(q, k, pos, freq, wq=wq, wk=wk, eps=EPS, interleaved=inter)
    for name, y, x, w in (("q", yq, q, wq), ("k", yk, k, wk)):
        ref, size = rope_ref(x, w, pos, freq, inter)
        within(f"{name} {n}x{x.shape[1]}x{D} rot {rot}", y, ref, ROPE * size, t)
    # rotation alone
    yq, yk = lb.lory_qk_rope(q, k, pos, freq, interleaved=inter)
    for name, y, x in (("q", yq, q), ("k", yk, k)):
        ref, size = rope_ref(x, None, pos, freq, inter)
        within(f"{name} without norm", y, ref, ROPE * size, t)
        assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("n,Hq,Hkv,D,rot,inter,dtype", [(7000, 24, 8, 128, 128, False, "f32"), (13001, 20, 5, 256, 64, True, "bf16")])
def test_rope_of_more_than_100_megabytes(n, Hq, Hkv, D, rot, inter, dtype):
    """Large calls are read another way; the store too."""
    g, t = gen(n), T[dtype]
    q, k, v = rnd(g, n, Hq, D, dtype=t), rnd(g, n, Hkv, D, dtype=t), rnd(g, n, Hkv, D, dtype=t)
    wq, wk = (1 + 0.3 * rnd(g, D)).to(t), (1 + 0.3 * rnd(g, D)).to(t)
    pos, freq = torch.randint(0, 5000, (n,), device="cuda", dtype=torch.int32), freqs(rot)
    w = dict(wq=wq, wk=wk, eps=EPS, interleaved=inter)
    yq, yk = lb.lory_qk_rope(q, k, pos, freq, **w)
    for name, y, x, wx in (("q", yq, q, wq), ("k", yk, k, wk)):
        ref, size = rope_ref(x, wx, pos, freq, inter)
        within(f"{name} {n}x{x.shape[1]}x{D}", y, ref, ROPE * size, t)
    page = 16
    kc, vc = (torch.zeros(-(-n // page), Hkv, page, D, device="cuda", dtype=t) for _ in range(2))
    slots = torch.randperm(kc.shape[0] * page, device="cuda")[:n]
    assert torch.equal(lb.lory_qk_rope_cache(q, k, v, pos, freq, kc, vc, slots, **w), yq)
    assert torch.equal(kc[slots // page, :, slots % page], yk) and torch.equal(vc[slots // page, :, slots % page], v)


def test_rope_strides_far_positions_and_in_place():
    g = gen(3)
    n, Hq, Hkv, D, rot = 37, 6, 2, 128, 128
    qkv = rnd(g, n, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    kt = k.transpose(0, 1).contiguous().transpose(0, 1)   # heads outside
    wq, wk = (rnd(g, D, dtype=torch.bfloat16) for _ in range(2))
    pos = torch.randint(0, 2 ** 31 - 1, (n,), device="cuda", dtype=torch.int32)
    pos[0], pos[1], pos[2] = 2 ** 31 - 1, -2 ** 31, 0
    freq = freqs(rot)
    yk = torch.empty(Hkv, n, D, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    yq, _ = lb.lory_qk_rope(q, kt, pos, freq, k_out=yk, wq=wq, wk=wk, eps=EPS)
    rq, sq = rope_ref(q, wq, pos, freq, False)
    rk, sk = rope_ref(k, wk, pos, freq, False)
    within("far q", yq, rq, ROPE * sq, torch.bfloat16)
    within("far k", yk, rk, ROPE * sk, torch.bfloat16)
    vv = v.clone()
    out = lb.lory_qk_rope(q, k, pos, freq, q_out=q, k_out=k, wq=wq, wk=wk, eps=EPS)
    assert out[0].data_ptr() == q.data_ptr() and torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(v, vv)


def test_rope_keeps_infinities_apart():
    """A value that is no number stays in its head, and without norm in its pair."""
    n, H, D, rot = 2, 3, 64, 32
    x = torch.ones(n, H, D, device="cuda")
    x[0, 1, 5], x[1, 2, 60], x[1, 0, 40] = float("nan"), float("inf"), float("-inf")
    pos, freq = torch.tensor([3, 9], device="cuda", dtype=torch.int32), freqs(rot)
    y, _ = lb.lory_qk_rope(x, x.clone(), pos, freq)
    ref, size = rope_ref(x, None, pos, freq, False)
    within("odd values", y, ref, torch.nan_to_num(ROPE * size, 0.0, 0.0), torch.float32)
    assert torch.isnan(y).sum() == 2 and torch.isinf(y).sum() == 2
    w = torch.ones(D, device="cuda")
    y, _ = lb.lory_qk_rope(x, x.clone(), pos, freq, wq=w, wk=w)
    bad = torch.zeros(n, H, dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 2] = bad[1, 0] = True
    assert torch.isfinite(y[~bad]).all() and torch.isnan(y[0, 1]).all()
    assert torch.isnan(y[1, 2, 60]) and (y[1, 2, :60] == 0).all()   # x / inf


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot", SHAPES + [(3000, 24, 8, 64, 64)])
def test_rope_gradient(n, Hq, Hkv, D, rot, inter, dtype):
    g = gen(n + D + 1)
    t = T[dtype]
    q, k = rnd(g, n, Hq, D, dtype=t), 3 * rnd(g, n, Hkv, D, dtype=t)
    dyq, dyk = rnd(g, n, Hq, D, dtype=t), rnd(g, n, Hkv, D, dtype=t)
    wq, wk = (1 + 0.3 * rnd(g, D)).to(t), (1 + 0.3 * rnd(g, D)).to(t)
    pos = torch.randint(-50, 5000, (n,), device="cuda", dtype=torch.int32)
    freq = freqs(rot)
    ws = lb.alloc_qk_rope_workspace(q, k)
    ws.fill_(255)   # NaN
    got = lb.lory_qk_rope_bwd(q, k, dyq, dyk, pos, freq, wq, wk, EPS, inter, workspace=ws)
    again = lb.lory_qk_rope_bwd(q, k, dyq, dyk, pos, freq, wq, wk, EPS, inter)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for name, x, w, dy, dx, dw in (("q", q, wq, dyq, got[0], got[2]), ("k", k, wk, dyk, got[1], got[3])):
        x, w, dy = x.double().requires_grad_(), w.double().requires_grad_(), dy.double()
        y, _ = rope_ref(x, w, pos, freq, inter)
        rx, rw = torch.autograd.grad(y, [x, w], dy)
        with torch.no_grad():
            r = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
            G = turned(dy, pos, freq, inter, magnitude=True)
            size = r * (G * w.abs() + x.abs() * r * r * (G * w.abs() * x.abs()).mean(-1, keepdim=True))
            # as y, with the second sum of the head, three more products and one addition
            within(f"d{name} {n}x{x.shape[1]}x{D} rot {rot}", dx, rx, 48 * E32 * size, t)
            # every addend as y; then one chain of additions: a lane's groups of its tokens, lanes, rows of partial sums
            chain = 24 + math.ceil(n / 4096) * (Hq + Hkv) + 6 + 3 + 1024 / 16 + 16
            within(f"dw{name}", dw, rw, chain * E32 * (G * x.abs() * r).sum((0, 1)))
    # rotation alone: the inputs are not read, and the gradient may replace its own
    nan = torch.full_like(q, float("nan"))
    dq, dk, dwq, dwk = lb.lory_qk_rope_bwd(nan, k, dyq.clone(), dyk, pos, freq, interleaved=inter)
    assert dwq is None and dwk is None
    within("dq without norm", dq, turned(dyq.double(), pos, freq, inter, sign=-1.0),
           ROPE * turned(dyq.double(), pos, freq, inter, magnitude=True), t)
    inplace = dyq.clone()
    d2 = lb.lory_qk_rope_bwd(q, k, inplace, dyk, pos, freq, wq, wk, EPS, inter, dq=inplace)
    assert d2[0] is inplace and torch.equal(inplace, got[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,D", [(1, 3, 1, 80), (5, 7, 3, 96), (16, 2, 1, 64), (17, 2, 1, 64), (16, 5, 1, 128), (2, 40, 2, 128),
                                        (1, 80, 5, 256), (16, 1, 1, 8)])
def test_rope_gradient_of_few_tokens(n, Hq, Hkv, D, dtype):
    """Tokens and bytes on both sides of where one workgroup takes them all."""
    test_rope_gradient(n, Hq, Hkv, D, D // 16 * 16, False, dtype)


def test_rope_gradient_against_differences():
    """Central differences of the operator's own forward: the truncation is h^2 / 6 of third derivatives of order 1, the
    rounding that of the 64 values that change, of order 2 with their gradient: 64 * 2 * 24 * 2^-24 / (2 h); with
    h = 2^-6 both stay below 2e-2."""
    g = gen(5)
    n, H, D, rot = 2, 3, 64, 32
    q, k, dy = rnd(g, n, H, D), rnd(g, n, 1, D), rnd(g, n, H, D)
    w = 1 + 0.3 * rnd(g, D)
    pos, freq = torch.tensor([3, 700], device="cuda", dtype=torch.int32), freqs(rot)

    def loss(q, w):
        return (lb.lory_qk_rope(q, k, pos, freq, wq=w, wk=w, eps=EPS)[0].double() * dy.double()).sum().item()

    dq, _, dw, _ = lb.lory_qk_rope_bwd(q, k, dy, torch.zeros_like(k), pos, freq, w, w, EPS)
    h = 2.0 ** -6
    for i in ((0, 0, 0), (0, 1, 17), (1, 2, 40), (1, 0, 63)):
        up, down = q.clone(), q.clone()
        up[i] += h
        down[i] -= h
        assert abs((loss(up, w) - loss(down, w)) / (2 * h) - dq[i].item()) < 2e-2
    for i in (0, 20, 63):
        up, down = w.clone(), w.clone()
        up[i] += h
        down[i] -= h
        assert abs((loss(q, up) - loss(q, down)) / (2 * h) - dw[i].item()) < 2e-2


def test_no_tokens():
    e = torch.empty(0, 4, 64, device="cuda")
    pos, freq, w = torch.empty(0, device="cuda", dtype=torch.int32), freqs(64), torch.ones(64, device="cuda")
    q, k = lb.lory_qk_rope(e, e, pos, freq, wq=w, wk=w)
    assert q.shape == e.shape and k.shape == e.shape
    dwq = torch.full((64,), float("nan"), device="cuda")
    _, _, dwq, dwk = lb.lory_qk_rope_bwd(e, e, e, e, pos, freq, w, w, dwq=dwq)
    assert (dwq == 0).all() and (dwk == 0).all()
    cache = torch.ones(2, 4, 16, 64, device="cuda")
    lb.lory_qk_rope_cache(e, e, e, pos, freq, cache, cache.clone(), torch.empty(0, device="cuda", dtype=torch.int64), wq=w, wk=w)
    assert (cache == 1).all()


# ---------------------------------------------------------------- store

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot,inter,page,norm", [(1, 4, 1, 64, 64, False, 16, True), (48, 32, 8, 128, 128, False, 16, True),
                                                             (301, 6, 3, 80, 32, True, 24, True), (9, 2, 2, 256, 64, False, 1, False),
                                                             (2000, 8, 2, 96, 96, True, 7, True), (5, 3, 1, 8, 0, False, 3, True)])
def test_store(n, Hq, Hkv, D, rot, inter, page, norm, dtype):
    g = gen(n)
    t = T[dtype]
    qkv = rnd(g, n, (Hq + 2 * Hkv) * D, dtype=t)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    w = dict(wq=(1 + 0.2 * rnd(g, D)).to(t), wk=(1 + 0.2 * rnd(g, D)).to(t)) if norm else {}
    pos = torch.randint(0, 9000, (n,), device="cuda", dtype=torch.int32)
    freq = freqs(rot)
    pages = -(-n // page) + 3
    slots = torch.randperm(pages * page, device="cuda")[:n].clone()
    if n > 4:   # no page of the cache: nothing is stored
        slots[1], slots[2], slots[3], slots[4] = -1, pages * page, 2 ** 62, -2 ** 63
    kc, vc = rnd(g, pages, Hkv, page, D, dtype=t), rnd(g, pages, Hkv, page, D, dtype=t)
    guard = [torch.cat([c.flatten(), torch.full((64,), 7.0, device="cuda", dtype=t)]) for c in (kc, vc)]
    kc2, vc2 = (x[:-64].view(pages, Hkv, page, D) for x in guard)
    yq, yk = lb.lory_qk_rope(q, k, pos, freq, eps=EPS, interleaved=inter, **w)
    out = lb.lory_qk_rope_cache(q, k, v, pos, freq, kc2, vc2, slots, eps=EPS, interleaved=inter, **w)
    assert torch.equal(out, yq)
    ok = (slots >= 0) & (slots < pages * page)
    p, r = slots[ok] // page, slots[ok] % page
    kc[p, :, r], vc[p, :, r] = yk[ok], v[ok]
    assert torch.equal(kc, kc2) and torch.equal(vc, vc2)
    assert all((x[-64:] == 7).all() for x in guard)


# ---------------------------------------------------------------- plan

def plan_oracle(lens, add, table, free, count, page, room):
    """The plan with lists; (status, ...) as lory_kv_plan describes it."""
    B, W = table.shape
    F = len(free)
    most = W * page
    ceil = lambda n: -(-n // page)
    status = 0
    n = [max(a, 0) for a in add]
    new = [0 if a < 0 else l + m for l, a, m in zip(lens, add, n)]
    if sum(n) > room:
        status |= 1
    if any(x > most for x in new):
        status |= 2
    if any(l < 0 or (a < 0 and l > most) for l, a in zip(lens, add)) or not 0 <= count <= F:
        status |= 16
    back = [ceil(max(l, 0)) if a < 0 else 0 for l, a in zip(lens, add)]
    take = [0 if a < 0 else ceil(max(l, 0) + m) - ceil(max(l, 0)) for l, a, m in zip(lens, add, n)]
    top = count + sum(back)
    status |= 4 * (sum(take) > top) | 8 * (top > F)
    positions, slots = [0] * room, [-1] * room
    table, free = table.copy(), list(free)
    if status:
        return dict(status=status, lens_new=lens, cu=[0] * (B + 1), count_new=count, positions=positions, slots=slots,
                    table=table, free=free)
    stack = free[:count]
    for b in range(B):
        stack += table[b, :back[b]].tolist()
    cu = [0]
    for b in range(B):
        for c in range(take[b]):
            table[b, ceil(lens[b]) + c] = stack.pop()
        for i in range(n[b]):
            at = lens[b] + i
            positions[cu[-1] + i] = at
            slots[cu[-1] + i] = int(table[b, at // page]) * page + at % page
        cu.append(cu[-1] + n[b])
    free[count:len(stack)] = stack[count:]
    return dict(status=0, lens_new=new, cu=cu, count_new=len(stack), positions=positions, slots=slots, table=table, free=free)


def run_plan(lens, add, table, free, count, page, room, wide=0):
    dev = lambda a, t=torch.int32: torch.tensor(np.asarray(a).tolist(), dtype=t, device="cuda")
    B, W = table.shape
    full = torch.full((B, W + wide), 99, dtype=torch.int32, device="cuda")
    full[:, :W] = dev(table)
    d = dict(lens=dev(lens), add=dev(add), table=full[:, :W], free=dev(free), count=dev([count]))
    o = dict(lens_new=dev([55] * B), cu=dev([55] * (B + 1)), positions=dev([55] * room), slots=dev([55] * room, torch.int64),
             count_new=dev([55]), status=dev([55]))
    call = lambda: lb.lory_kv_plan(d["lens"], d["add"], d["table"], d["free"], d["count"], page, o["lens_new"], o["cu"],
                                   o["positions"], o["slots"], o["count_new"], o["status"])
    assert call() is o["status"]
    got = {**{k: v.clone() for k, v in o.items()}, "table": d["table"].clone(), "free": d["free"].clone()}
    call()   # the same plan again
    for k, v in {**o, "table": d["table"], "free": d["free"]}.items():
        assert torch.equal(v, got[k]), k
    assert (full[:, W:] == 99).all()
    return got


def check_plan(*args, wide=0):
    ref, got = plan_oracle(*args), run_plan(*args, wide=wide)
    for k, v in ref.items():
        v = torch.tensor([v] if isinstance(v, int) else np.asarray(v).tolist(), dtype=torch.int64)
        assert torch.equal(got[k].cpu().long().reshape(-1), v.reshape(-1)), k
    return ref["status"]


def plan_state(rs, B, page, hi, extra=5, p_end=0.2, p_new=0.3, new=40):
    lens = rs.randint(0, hi + 1, B)
    add = np.where(rs.rand(B) < p_end, -1 - rs.randint(0, 3, B), np.where(rs.rand(B) < p_new, rs.randint(0, new + 1, B), 1))
    blocks = -(-lens // page)
    W = int((-(-(lens + np.maximum(add, 0)) // page)).max(initial=0)) + 1
    total = int(blocks.sum()) + int((-(-(lens + np.maximum(add, 0)) // page) - blocks).clip(0).sum()) + extra
    perm = rs.permutation(total)
    table = np.full((B, W), -1)
    table[np.arange(W)[None] < blocks[:, None]] = perm[:blocks.sum()]
    free = np.full(total, -1)
    count = total - int(blocks.sum())
    free[:count] = perm[blocks.sum():]
    room = int(np.maximum(add, 0).sum()) + 3
    return lens.tolist(), add.tolist(), table, free.tolist(), count, page, room


@pytest.mark.parametrize("B,page,hi,new", [(1, 16, 0, 1), (1, 1, 5, 3), (7, 16, 100, 40), (64, 24, 300, 70), (512, 16, 50, 9),
                                           (513, 7, 60, 30), (1025, 32, 90, 100), (1600, 5, 20, 2)])
@pytest.mark.parametrize("p_end", [0.0, 0.3, 1.0])
def test_plan(B, page, hi, new, p_end):
    rs = np.random.RandomState(B + page)
    state = plan_state(rs, B, page, hi, p_end=p_end, new=new)
    assert check_plan(*state, wide=3 * (B % 2)) == 0


def test_plan_takes_pages_that_come_back():
    """No free page at the start: what the ended rows give is what the others get, from the last row's last page down."""
    table = np.array([[3, 1, 4, -1], [0, -1, -1, -1], [2, 5, -1, -1]])
    got = run_plan([33, 16, 17], [-1, 18, -2], table, [-1] * 6, 0, 16, 20)
    assert got["table"][1].tolist() == [0, 5, 2, -1] and got["count_new"].item() == 3
    assert got["free"].tolist() == [3, 1, 4, -1, -1, -1] and got["lens_new"].tolist() == [0, 34, 0]
    assert check_plan([33, 16, 17], [-1, 18, -2], table, [-1] * 6, 0, 16, 20) == 0


@pytest.mark.parametrize("change,status", [(dict(room=-1), 1), (dict(lens0=16 * 4 - 1, add0=2), 2), (dict(count=2), 4),
                                           (dict(count=9, end=True), 8), (dict(lens0=-3), 16), (dict(count=-1), 16 + 4),
                                           (dict(count=10), 16 + 8), (dict(lens0=65, add0=-1), 16),
                                           (dict(lens0=2 ** 31 - 1, add0=2 ** 31 - 1), 1 + 2 + 4)])
def test_plan_status(change, status):
    table = np.array([[0, 1, 2, 3], [4, -1, -1, -1]])
    lens, add, free, count = [60, 16], [4, 33], [8, 7, 6, 5] + [-1] * 5, 4
    room = 37 + change.get("room", 0)
    lens[0], add[0] = change.get("lens0", 60), change.get("add0", 4)
    count = change.get("count", count)
    if change.get("end"):
        add[1] = -1
    assert plan_oracle(lens, add, table, free, count, 16, room)["status"] == status
    assert check_plan(lens, add, table, free, count, 16, room) == status


def test_plan_without_rows():
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    one = lambda v: torch.tensor([v], dtype=torch.int32, device="cuda")
    free, cu, cn, st = one(3), one(9), one(9), one(9)
    pos, slots = torch.full((5,), 9, dtype=torch.int32, device="cuda"), torch.full((5,), 9, device="cuda")
    lb.lory_kv_plan(e, e, torch.empty(0, 4, dtype=torch.int32, device="cuda"), free, one(1), 16, e, cu, pos, slots, cn, st)
    assert cu.item() == 0 and cn.item() == 1 and st.item() == 0 and (pos == 0).all() and (slots == -1).all()


# ---------------------------------------------------------------- attention

def paged_case(seed, lens, Hq, Hkv, D, page, dtype, width=None, sigma=2.0, least_bytes=0):
    """q, caches whose unused places hold NaN and infinities, a table whose unused entries are no pages."""
    g = gen(seed)
    t = T[dtype]
    lens = np.asarray(lens)
    blocks = -(-lens // page)
    W = width or max(1, int(blocks.max(initial=0)))
    total = int(blocks.sum()) + 3
    while 2 * total * Hkv * page * D * t.itemsize <= least_bytes:
        total *= 2
    perm = np.random.RandomState(seed).permutation(total)
    table = np.random.RandomState(seed + 1).choice([-1, total, 2 ** 31 - 1, -2 ** 31, 10 ** 6], size=(len(lens), W))
    table[np.arange(W)[None] < blocks[:, None]] = perm[:blocks.sum()]
    k, v = rnd(g, total, Hkv, page, D, dtype=t), rnd(g, total, Hkv, page, D, dtype=t)
    used = torch.zeros(total, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        for c in range(int(blocks[b])):
            used[table[b, c], :min(page, n - c * page)] = True
    used = used.cuda()[:, None, :, None]
    junk = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(t)
    fill = junk[torch.arange(page, device="cuda") % 3][None, None, :, None]
    k, v = torch.where(used, k, fill), torch.where(used, v, fill)
    q = rnd(g, len(lens), Hq, D) * sigma
    i32 = lambda a: torch.from_numpy(np.asarray(a)).to(dtype=torch.int32, device="cuda")
    return q.to(t), k, v, i32(table), i32(lens)


def check_attention(label, out, lse, q, k, v, table, lens, scale=None, skip=None):
    """skip[b]: tokens left out of row b."""
    t = out.dtype
    B, Hq, D = q.shape
    Hkv, page = k.shape[1], k.shape[2]
    g = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    ref, size = torch.zeros(B, Hq, D, dtype=torch.float64, device="cuda"), torch.zeros(B, Hq, D, dtype=torch.float64, device="cuda")
    rlse = torch.full((B, Hq), float("-inf"), dtype=torch.float64, device="cuda")
    bound, lbound = torch.zeros_like(ref), torch.zeros_like(rlse)
    for b, n in enumerate(lens.tolist()):
        keep = [i for i in range(n) if skip is None or i not in skip.get(b, ())]
        if not keep:
            continue
        keep = torch.tensor(keep, device="cuda")
        pages = table[b].long()[keep // page]
        for h in range(Hkv):
            K, V = k[pages, h, keep % page].double(), v[pages, h, keep % page].double()
            Q = q[b, h * g:(h + 1) * g].double()
            z = Q @ K.T * scale
            # a score: D products and additions, the scale and the base of the logarithm (4 more), its maximum taken off (2)
            dz = (Q.abs() @ K.abs().T * scale).amax(-1) * (D + 6) * E32
            p = torch.softmax(z, -1)
            s = slice(h * g, (h + 1) * g)
            ref[b, s] = p @ V
            rlse[b, s] = torch.logsumexp(z, -1)
            # probabilities: both sums carry dz and the exponential (4); two bf16 terms 2^-16; one chain of additions: a
            # wavefront's steps of 16 keys at least, wavefronts, pieces, lanes
            chain = n / 16 + 64
            rel = 2 * dz + (4 + 2 * chain) * E32 + (2.0 ** -16 if t == torch.bfloat16 else 0.0)
            bound[b, s] = rel[:, None] * (p @ V.abs())
            lbound[b, s] = dz + (4 + chain) * E32 + 4 * E32 * rlse[b, s].abs()
    within(f"{label} out", out, ref, bound, t)
    within(f"{label} lse", lse, rlse, lbound)


def same(a, b):
    """Equal bit for bit, NaN included."""
    i = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(i), b.contiguous().view(i))


def attend(case, **kw):
    q, k, v, table, lens = case
    lse = torch.full(q.shape[:2], 77.0, device="cuda")
    ws = lb.alloc_paged_attn_workspace(q, k, table)
    ws.fill_(255)
    out = lb.lory_paged_attn(q, k, v, table, lens, lse=lse, workspace=ws, **kw)
    lse2 = torch.empty_like(lse)
    assert same(out, lb.lory_paged_attn(q, k, v, table, lens, lse=lse2, **kw)) and same(lse, lse2)
    assert same(out, lb.lory_paged_attn(q, k, v, table, lens, **kw))   # without lse
    return out, lse


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 0, 2]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,page", [(1, 1, 64, 16), (4, 4, 64, 8), (8, 2, 128, 16), (5, 1, 80, 24), (15, 3, 96, 32),
                                           (16, 1, 128, 64), (17, 1, 64, 16), (40, 1, 128, 128), (6, 2, 256, 16), (8, 8, 8, 1),
                                           (2, 1, 40, 7), (3, 3, 200, 5), (20, 4, 80, 24), (8, 1, 136, 1000), (7, 1, 24, 3)])
def test_attention(Hq, Hkv, D, page, dtype):
    case = paged_case(Hq + D, LENS, Hq, Hkv, D, page, dtype)
    check_attention(f"{Hq}/{Hkv}x{D} page {page}", *attend(case), *case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,Hq,Hkv,D,page", [([1], 2, 1, 64, 16), ([0], 4, 2, 128, 16), ([0, 0, 0], 4, 2, 64, 16),
                                                ([3000, 2999, 1], 12, 4, 128, 16), ([20011], 2, 1, 64, 64),
                                                ([70001, 3], 4, 2, 64, 128), ([9000] + [5] * 40, 4, 1, 128, 16)])
def test_attention_split_over_the_cache(lens, Hq, Hkv, D, page, dtype):
    case = paged_case(len(lens) + D, lens, Hq, Hkv, D, page, dtype)
    check_attention(f"{lens[:3]} {Hq}/{Hkv}x{D}", *attend(case), *case)


@pytest.mark.parametrize("B", [255, 257, 700])
def test_attention_many_rows(B):
    lens = np.random.RandomState(B).randint(0, 90, B)
    case = paged_case(B, lens, 4, 2, 64, 16, "bf16")
    check_attention(f"{B} rows", *attend(case), *case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,Hq,Hkv,D,page", [([0, 1, 31, 300, 65], 8, 2, 64, 16), ([5000, 3, 129], 12, 4, 128, 16),
                                                ([700, 64], 3, 1, 40, 8), ([333, 4000], 20, 4, 80, 24), ([77, 2100], 6, 2, 256, 16),
                                                ([90, 500], 17, 1, 200, 32)])
def test_attention_of_a_large_cache(lens, Hq, Hkv, D, page, dtype):
    """Caches of more than 64 MB are read another way."""
    case = paged_case(len(lens) + D, lens, Hq, Hkv, D, page, dtype, least_bytes=64 << 20)
    check_attention(f"large cache {lens[:3]} {Hq}/{Hkv}x{D}", *attend(case), *case)


@pytest.mark.parametrize("wide", [False, True])
def test_attention_of_more_rows_than_a_grid_dimension(wide):
    """70000 rows of up to four tokens, in one launch or (a table that allows long rows, and three long ones) in ranges."""
    B, D, page, W = 70000, 8, 4096 if wide else 4, 8 if wide else 1
    g = gen(3)
    lens = torch.randint(0, 5, (B,), generator=g, device="cuda", dtype=torch.int32)
    pages = 24 if wide else 1000
    k, v = rnd(g, pages, 1, page, D), rnd(g, pages, 1, page, D)
    table = torch.randint(0, pages, (B, W), generator=g, device="cuda", dtype=torch.int32)
    q = rnd(g, B, 1, D)
    long = {17: 9000, 40000: 32768, B - 1: 4097} if wide else {}
    for b, n in long.items():
        lens[b] = n
    lse = torch.empty(B, 1, device="cuda")
    out = lb.lory_paged_attn(q, k, v, table, lens, lse=lse)
    short = torch.ones(B, dtype=torch.bool, device="cuda")
    short[list(long)] = False
    here = torch.arange(4, device="cuda") < lens[:, None]
    K, V = (x[table[:, 0].long(), 0, :4].double() for x in (k, v))
    z = (K * q.double()).sum(-1) * D ** -0.5
    z = torch.where(here, z, float("-inf"))
    p = torch.softmax(z, -1).nan_to_num(0.0)
    # as in check_attention: scores of D terms, one chain of additions
    dz = (K.abs() * q.double().abs()).sum(-1).amax(-1) * D ** -0.5 * (D + 6) * E32
    rel = (2 * dz + (4 + 2 * 65) * E32)[:, None]
    ref, bound = (p[..., None] * V).sum(1), rel * (p[..., None] * V.abs()).sum(1)
    within("many rows", out[short, 0], ref[short], bound[short], torch.float32)
    rl = torch.logsumexp(z, -1)
    within("many rows lse", lse[short, 0], rl[short], (dz + 80 * E32 + 4 * E32 * rl.abs().nan_to_num(0.0, 0.0))[short])
    for b in long:
        check_attention(f"long row {b}", out[b:b + 1], lse[b:b + 1], q[b:b + 1], k, v, table[b:b + 1], lens[b:b + 1])


def test_attention_strides_scale_and_in_place():
    Hq, Hkv, D, page = 6, 2, 128, 16
    q, k, v, table, lens = paged_case(2, [40, 0, 333, 7], Hq, Hkv, D, page, "bf16")
    wide = torch.full((4, (Hq + 4) * D), 5.0, device="cuda", dtype=torch.bfloat16)
    qs = wide[:, :Hq * D].unflatten(1, (Hq, D))
    qs.copy_(q)
    tall = torch.full((4, table.shape[1] + 9), -7, device="cuda", dtype=torch.int32)
    tall[:, :table.shape[1]] = table
    view = tall[:, :table.shape[1]]
    want, lse = attend((q, k, v, table, lens), scale=0.3)
    check_attention("scale", want, lse, q, k, v, table, lens, scale=0.3)
    outside = torch.empty(Hq, 4, D, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    assert torch.equal(lb.lory_paged_attn(qs, k, v, view, lens, out=outside, scale=0.3), want)
    assert lb.lory_paged_attn(qs, k, v, view, lens, out=qs, scale=0.3) is qs and torch.equal(qs, want)
    assert (wide[:, Hq * D:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_leaves_out_what_has_no_page(dtype):
    lens, page = [100, 40, 16, 900], 16
    case = paged_case(9, lens, 4, 2, 64, page, dtype)
    q, k, v, table, dlens = case
    table = table.clone()
    table[0, 2], table[1, 0], table[2, 0], table[3, 56] = -1, k.shape[0], 2 ** 31 - 1, -2 ** 31
    table[3, 10:20] = -5
    skip = {0: range(32, 48), 1: range(16), 2: range(16), 3: list(range(160, 320)) + list(range(896, 912))}
    case = (q, k, v, table, dlens)
    check_attention("bad pages", *attend(case), *case, skip=skip)


def test_attention_bounds_lengths():
    """Lengths below 0 count as 0, those above the table as all of it."""
    q, k, v, table, lens = paged_case(4, [48, 48, 20], 2, 2, 64, 16, "bf16")
    out, lse = attend((q, k, v, table, torch.tensor([-5, 2 ** 31 - 1, 20], device="cuda", dtype=torch.int32)))
    check_attention("lengths", out, lse, q, k, v, table, torch.tensor([0, 48, 20], device="cuda", dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_extreme_scores(dtype):
    """Heads whose scores are all -inf give 0 and -inf; lowest values and large scores stay exact; NaN stays in its head."""
    t = T[dtype]
    q, k, v, table, lens = paged_case(6, [200, 200, 200, 200], 2, 2, 64, 16, dtype, sigma=1.0)
    k, v = k.clone(), v.clone()
    p0, p1, p2, p3 = (table[i].long()[:13] for i in range(4))
    q[0] = q[0].abs() + 0.1
    k[p0, 0] = float("-inf")                       # row 0, head 0: nothing counts
    q[1], k[p1, 0] = 0, 0
    q[1, 0, 0] = 1.0
    k[p1, 0, :, 0] = torch.finfo(t).min            # row 1, head 0: every score the lowest value, all alike
    q[2] = q[2] * 100                              # scores of hundreds: one key takes all
    v[p3[3], 1, 5, 7] = float("nan")               # row 3, head 1, one value
    out, lse = attend((q, k, v, table, lens))
    assert (out[0, 0] == 0).all() and lse[0, 0] == float("-inf") and torch.isfinite(out[0, 1]).all()
    mean = torch.cat([v[p1, 0].reshape(-1, 64)[:200]]).double().mean(0)
    within("lowest", out[1, 0], mean, (2.0 ** -16 + 200 * E32) * torch.ones_like(mean), t)
    assert abs(lse[1, 0].item() / (torch.finfo(t).min / 8) - 1) < 8 * E32
    assert torch.isnan(out[3, 1, 7]) and torch.isnan(out).sum() == 1
    keep = [(0, 1), (2, 0), (2, 1), (3, 0)]
    kk, vv = k.clone(), v.clone()
    kk[p0, 0], vv[p3[3], 1, 5, 7] = 0, 0
    ref_out, ref_lse = attend((q, kk, vv, table, lens))
    for b, h in keep:
        assert torch.equal(out[b, h], ref_out[b, h]) and lse[b, h] == ref_lse[b, h]
    check_attention("large", ref_out[2:3], ref_lse[2:3], q[2:3], kk, vv, table[2:3], lens[2:3])


def test_attention_cache_above_32_bits():
    """Rows of a cache of more than 2^32 bytes, on both sides of the limits of 31 and 32 bits."""
    Hq, Hkv, D, page = 4, 2, 128, 64
    pages = (1 << 33) // (Hkv * page * D * 2) + 70
    k, v = (torch.empty(pages, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    g = gen(1)
    per = Hkv * page * D * 2
    ids = [0, (1 << 31) // per - 1, (1 << 31) // per, (1 << 32) // per - 1, (1 << 32) // per, (1 << 33) // per, pages - 1]
    for i in ids:
        k[i], v[i] = rnd(g, Hkv, page, D).bfloat16(), rnd(g, Hkv, page, D).bfloat16()
    q = rnd(g, 2, Hq, D, dtype=torch.bfloat16)
    table = torch.tensor([ids, ids[::-1]], device="cuda", dtype=torch.int32)
    lens = torch.tensor([7 * page, 6 * page + 5], device="cuda", dtype=torch.int32)
    check_attention("far pages", *attend((q, k, v, table, lens)), q, k, v, table, lens)
    # and the store
    n = 3
    x = rnd(g, n, Hkv, D, dtype=torch.bfloat16)
    slots = torch.tensor([pages * page - 1, ((1 << 32) // per) * page + 1, 5], device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    lb.lory_qk_rope_cache(rnd(g, n, Hq, D, dtype=torch.bfloat16), x, x, pos, freqs(D), k, v, slots)
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(k[s // page, :, s % page], x[i]) and torch.equal(v[s // page, :, s % page], x[i])


def test_on_another_stream_and_in_a_graph():
    """A whole step (plan, store, attention) on a side stream, then captured and replayed with the program's own work between
    the replays; every replay against the same step run eagerly."""
    Hq, Hkv, D, page, B, W, F = 8, 2, 64, 16, 5, 20, 120
    g = gen(8)
    rs = np.random.RandomState(8)
    freq, w = freqs(D), torch.ones(D, device="cuda", dtype=torch.bfloat16)
    i32 = lambda a: torch.tensor(np.asarray(a).tolist(), dtype=torch.int32, device="cuda")

    class Step:
        def __init__(self):
            self.lens, self.add, self.count = i32([0] * B), i32([0] * B), i32([F])
            self.table, self.free = i32(np.full((B, W), -1)), i32(range(F))
            self.lens_new, self.cu, self.count_new, self.status = i32([0] * B), i32([0] * (B + 1)), i32([0]), i32([0])
            self.positions, self.slots = i32([0] * B), torch.zeros(B, dtype=torch.int64, device="cuda")
            self.k, self.v = (torch.zeros(F, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            self.qkv = torch.zeros(B, (Hq + 2 * Hkv) * D, device="cuda", dtype=torch.bfloat16)
            self.q, self.kx, self.vx = (x.unflatten(1, (-1, D)) for x in self.qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
            self.y = torch.empty(B, Hq, D, device="cuda", dtype=torch.bfloat16)
            self.out, self.lse = torch.empty_like(self.y), torch.empty(B, Hq, device="cuda")
            self.ws = lb.alloc_paged_attn_workspace(self.q, self.k, self.table)

        def run(self):
            lb.lory_kv_plan(self.lens, self.add, self.table, self.free, self.count, page, self.lens_new, self.cu,
                            self.positions, self.slots, self.count_new, self.status)
            lb.lory_qk_rope_cache(self.q, self.kx, self.vx, self.positions, freq, self.k, self.v, self.slots, q_out=self.y,
                                  wq=w, wk=w)
            lb.lory_paged_attn(self.y, self.k, self.v, self.table, self.lens_new, out=self.out, lse=self.lse, workspace=self.ws)
            self.lens.copy_(self.lens_new)
            self.count.copy_(self.count_new)

    eager, side, captured = Step(), Step(), Step()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    Step().run()
    with torch.cuda.graph(graph):
        captured.run()
    for i in range(25):
        add = np.where(rs.rand(B) < 0.15, -1, 1)
        qkv = rnd(g, B, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16)
        for s in (eager, side, captured):
            s.add.copy_(i32(add))
            s.qkv.copy_(qkv)
        eager.run()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            side.run()
        torch.cuda.current_stream().wait_stream(stream)
        graph.replay()
        junk = torch.randn(1000, 1000, device="cuda")
        (junk @ junk).sum().item()
        assert eager.status.item() == 0
        for s in (side, captured):
            for n in ("lens", "count", "table", "free", "cu", "positions", "slots", "status", "k", "v", "y", "out", "lse"):
                assert torch.equal(getattr(s, n), getattr(eager, n)), (i, n)
    n = eager.lens.tolist()
    # rows that have just ended keep stale pages in the table; their length is 0
    check_attention("last step", eager.out, eager.lse, eager.y, eager.k, eager.v, eager.table.clamp(min=0), eager.lens)
    assert max(n) > 5


def test_event_timing_knows_the_operators():
    n, H, D, page = 64, 4, 64, 16
    x, pos, freq, w = rnd(gen(0), n, H, D), torch.zeros(n, dtype=torch.int32, device="cuda"), freqs(D), torch.ones(D, device="cuda")
    cache = torch.zeros(8, H, page, D, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    lb.lory_profile_read()
    lb.lory_profile_enable(True)
    try:
        lb.lory_qk_rope(x, x, pos, freq)
        lb.lory_qk_rope_bwd(x, x, x, x, pos, freq, w, w)
        lb.lory_paged_attn(x, cache, cache, torch.zeros(n, 1, dtype=torch.int32, device="cuda"), pos)
        lb.lory_kv_plan(i32(0), i32(1), i32(0)[None], i32(0), i32(1), 16, i32(0), i32(0, 0), i32(0), torch.zeros(1, dtype=torch.int64, device="cuda"),
                        i32(0), i32(0))
        got = {s["name"]: s for s in lb.lory_profile_read()}
    finally:
        lb.lory_profile_enable(False)
    assert set(got) == {"qk_rope", "qk_rope_bwd", "kv_plan", "paged_attn"}
    assert all(s["launches"] == 1 and s["ms"] > 0 for s in got.values())
    assert got["qk_rope"]["bytes"] == 4 * n * 2 * H * D * 4 // 2 + 4 * n and got["qk_rope_bwd"]["bytes"] == 3 * 4 * n * 2 * H * D + 4 * n


# ---------------------------------------------------------------- under autograd, and all together

def test_autograd_of_norm_and_rotation():
    """Leaves of one product, shared heads by expansion, an output that is not used: against autograd of the formula."""
    from paper_2405_03133_amd.autograd import qk_rope
    g = gen(12)
    n, Hq, Hkv, D = 19, 6, 2, 64
    base = rnd(g, n, (Hq + Hkv) * D)
    wq, wk = 1 + 0.3 * rnd(g, D), 1 + 0.3 * rnd(g, D)
    pos, freq = torch.randint(0, 999, (n,), device="cuda", dtype=torch.int32), freqs(D)
    c = rnd(g, n, Hq, D)

    def grads(f, dtype, only_q, shared):
        x, a, b = (t.to(dtype).requires_grad_() for t in (base, wq, wk))
        q, k = (t.unflatten(1, (-1, D)) for t in x.split([Hq * D, Hkv * D], 1))
        if shared:
            q = q[:, :1].expand(n, Hq, D)
        yq, yk = f(q, k, a, b)
        loss = (yq * c.to(dtype)).sum()
        if not only_q:
            loss = loss + yk.sum()   # its gradient is an expanded one
        return torch.autograd.grad(loss, [x, a, b], allow_unused=True)

    def formula(q, k, a, b):
        f = lambda x, w: turned(x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w, pos, freq, False)
        return f(q, a), f(k, b)

    for only_q in (False, True):
        for shared in (False, True):
            got = grads(lambda q, k, a, b: qk_rope(q, k, pos, freq, a, b, EPS), torch.float32, only_q, shared)
            ref = grads(formula, torch.float64, only_q, shared)
            for name, a, b in zip(("x", "wq", "wk"), got, ref):
                b = torch.zeros_like(a, dtype=torch.float64) if b is None else b
                # sums of up to 6 * 19 terms of order 1, 48 * 2^-24 of each
                assert (a.double() - b).abs().max().item() <= 48 * E32 * 114 * max(1.0, b.abs().max().item()), (name, only_q, shared)


def test_generation_example():
    """The example's block over prompts of different lengths and eight steps in which one request ends, in fp32 against the
    same block in 64 bits (the bars of the layer's fp32 configuration)."""
    import importlib.util
    import os

    from parity_util import check, host
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate_block.py")
    spec = importlib.util.spec_from_file_location("generate_block", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    block = ex.Block(d=128, heads=6, kv_heads=2, head_dim=64, d_ff=192, experts=4, dtype=torch.float32)
    B, L, steps, page = 5, 37, 8, 8
    requests = ex.Requests(block, B, B * 6, page, L + steps)
    lens = torch.tensor([37, 1, 8, 20, 9], device="cuda", dtype=torch.int32)
    prompts = rnd(gen(21), B, L, block.d)

    W = {n: getattr(block, n).double() for n in ("Wqkv", "Wo", "wq", "wk", "R", "Wg", "Wu", "Wd")}
    H, Hkv, D = block.H, block.Hkv, block.D

    def ffn(x, m):
        a, b = x @ m[0], x @ m[1]
        return (a * torch.sigmoid(a) * b) @ m[2]

    def plain(x, past, m):
        """Tokens x [n, d] behind the request's cached (k, v); all in 64 bits."""
        n, at = x.shape[0], 0 if past is None else past[0].shape[0]
        q, k, v = (t.unflatten(1, (-1, D)) for t in (x @ W["Wqkv"]).split([H * D, Hkv * D, Hkv * D], 1))
        pos = torch.arange(at, at + n, device="cuda")
        norm = lambda t, w: turned(t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w, pos, block.freq, False)
        q, k = norm(q, W["wq"]), norm(k, W["wk"])
        if past is not None:
            k, v = torch.cat([past[0], k]), torch.cat([past[1], v])
        out = torch.empty(n, H, D, dtype=torch.float64, device="cuda")
        for h in range(H):
            z = q[:, h] @ k[:, h // 3].T * D ** -0.5
            z = z.masked_fill(torch.arange(at + n, device="cuda")[None] > pos[:, None], float("-inf"))
            out[:, h] = torch.softmax(z, -1) @ v[:, h // 3]
        y = x + out.flatten(1) @ W["Wo"]
        return y + ffn(y, m), (k, v)

    h, merged = ex.prefill(block, requests, prompts, lens)
    ref, x64 = [], []
    for b, n in enumerate(lens.tolist()):
        e = torch.softmax(prompts[b, :n].double().mean(0) @ W["R"], -1)
        m = [torch.tensordot(e, W[k], 1) for k in ("Wg", "Wu", "Wd")]
        y, past = plain(prompts[b, :n].double(), None, m)
        check(f"prompt of {n}", host(h[b, :n]), y.cpu().numpy(), 1e-5)
        ref.append((past, m))
    x = ex.next_input(h[torch.arange(B, device="cuda"), lens.long() - 1])
    active = torch.ones(B, dtype=torch.bool, device="cuda")
    for step in range(steps):
        if step == 4:
            active[2] = False
        out = ex.decode(block, requests, x, active, merged)
        for b in range(B):
            if active[b]:
                y, past = plain(x[b:b + 1].double(), ref[b][0], ref[b][1])
                check(f"step {step} request {b}", host(out[b:b + 1]), y.cpu().numpy(), 1e-5)
                ref[b] = (past, ref[b][1])
        x = torch.where(active[:, None], ex.next_input(out), x)
    assert requests.lens.tolist() == [45, 9, 0, 28, 17] and requests.status.item() == 0
    assert requests.count.item() == B * 6 - (6 + 2 + 4 + 3)
