"""The attention half of a generating (or training) block: what its operators cost.

Three operators around a paged key-value cache, as a program that generates with merged experts runs
them in every block, and their training form: the plan of a step (pages, slots and positions from the
requests' lengths), the norms of the query and key heads with the position rotation (alone, with its
backward pass, or together with the store into the cache), and the attention of one new token per
request over the cache.  Head counts are those of the widths that `paper_2405_03133_amd.inputs.CONFIGS`
has (1024, 1536, 2048, 4096) with heads of 64 or 128, some of them with shared key-value heads.

`own` chooses between the plain forms below (elementary torch operations in 32 bits) and the calls of
`paper_2405_03133_amd.binding`.
"""
import math

import numpy as np
import torch

own = False


def _case(name, kind, **kw):
    return {"name": name, "kind": kind, **kw}


def listed():
    return [
        # one decode step of a small batch: one new token a request, latency only
        _case("plan_decode", "plan", B=64, lo=17, hi=4096, page=16, mixed=False, prompt=0),
        # a step of a busy server: most requests decode, every eighth has ended, every eighth starts with its prompt
        _case("plan_mixed", "plan", B=1000, lo=100, hi=6000, page=32, mixed=True, prompt=2048),
        # queries and keys of one training step at the headline width: 4 sequences of 4096 tokens, 16 heads of 128
        _case("rope_train", "rope", dtype="bf16", tokens=16384, Hq=16, Hkv=16, D=128, rot=128, pairs=False, far=4096),
        # fp32, shared heads of 80 of which 32 turn, neighbouring pairs, a token count without factors
        _case("rope_odd_f32", "rope", dtype="f32", tokens=4093, Hq=12, Hkv=4, D=80, rot=32, pairs=True, far=4093),
        # the gradient of the headline width's step
        _case("bwd_train", "bwd", dtype="bf16", tokens=16384, Hq=16, Hkv=16, D=128, rot=128, pairs=False, far=4096),
        # fp32 gradient of the 1536 width with heads of 64, eight of them shared, neighbouring pairs
        _case("bwd_gqa_f32", "bwd", dtype="f32", tokens=2999, Hq=24, Hkv=8, D=64, rot=64, pairs=True, far=2999),
        # the new tokens of a decode step go into the cache, at positions far into long requests
        _case("store_decode", "store", dtype="bf16", tokens=48, Hq=32, Hkv=8, D=128, rot=128, pairs=False, page=16,
              far=500000),
        # the prompts of a step go into the cache
        _case("store_prompt", "store", dtype="bf16", tokens=12001, Hq=16, Hkv=4, D=128, rot=128, pairs=False, page=16,
              far=12001),
        # one request at the 0.3B width (16 heads of 64) after a thousand tokens: latency
        _case("attn_b1", "attn", dtype="bf16", B=1, lo=1000, hi=1000, none=0, Hq=16, Hkv=16, D=64, page=16),
        # a batch of very different lengths with shared heads; one row is idle
        _case("attn_ragged", "attn", dtype="bf16", B=48, lo=1, hi=9000, none=1, Hq=16, Hkv=4, D=128, page=16),
        # four long contexts at the 4096 width
        _case("attn_long", "attn", dtype="bf16", B=4, lo=50000, hi=131072, none=0, Hq=32, Hkv=8, D=128, page=64),
        # fp32, groups of five heads of 80, pages that are no power of two, idle rows
        _case("attn_f32_odd", "attn", dtype="f32", B=7, lo=3, hi=3001, none=2, Hq=20, Hkv=4, D=80, page=24),
    ]


# ---------------------------------------------------------------- drawn cases

def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def _heads(rng, c):
    c["D"] = rng.choice([64, 128, 128, 128, 80, 96, 256])
    c["Hkv"] = rng.choice([1, 2, 4, 4, 8, 8, 16])
    c["Hq"] = c["Hkv"] * rng.choice([1, 2, 3, 4, 4, 5, 8] if c["Hkv"] <= 8 else [1, 2])
    return c


_LARGEST_BYTES = 2 * 4 * 131072 * 8 * 128 * 2


def draw(rng):
    kind = rng.choice(["plan", "rope", "bwd", "store", "attn", "attn"])
    while True:
        c = {"kind": kind}
        if kind == "plan":
            c.update(B=_log(rng, 1, 2048), lo=_log(rng, 1, 300), page=rng.choice([8, 16, 16, 24, 32, 64, 128]))
            c["hi"] = c["lo"] + _log(rng, 1, 8000)
            c["mixed"] = rng.random() < 0.6
            c["prompt"] = _log(rng, 20, 4096) if c["mixed"] else 0
            return c
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        _heads(rng, c)
        e = _esize(c)
        if kind == "attn":
            c["B"] = _log(rng, 1, 200)
            c["hi"] = _log(rng, 1, 131072)
            c["lo"] = rng.choice([c["hi"], max(1, c["hi"] // 3), 1])
            c["none"] = rng.choice([0, 0, 1]) if c["B"] > 1 else 0
            c["page"] = rng.choice([8, 16, 16, 24, 32, 64, 128])
            if 2 * c["B"] * c["hi"] * c["Hkv"] * c["D"] * e <= _LARGEST_BYTES // 2:
                return c
        else:
            c["rot"] = rng.choice([c["D"], c["D"], c["D"], 32])
            c["pairs"] = rng.random() < 0.4
            c["tokens"] = _log(rng, 1, 20000)
            c["far"] = rng.choice([c["tokens"], 4096, 131072, 1000000])
            if kind == "store":
                c["page"] = rng.choice([8, 16, 16, 24, 32, 64, 128])
            if 3 * c["tokens"] * (c["Hq"] + 2 * c["Hkv"]) * c["D"] * e <= _LARGEST_BYTES // 4:
                return c


# ---------------------------------------------------------------- inputs

def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _spread(n, lo, hi):
    """n lengths from lo to hi, even over their logarithm."""
    return np.rint(np.exp(np.linspace(math.log(lo), math.log(hi), n))).astype(np.int64) if n > 1 else np.array([hi] * n)


def _lengths(c):
    return np.concatenate([np.zeros(c["none"], np.int64), _spread(c["B"] - c["none"], c["lo"], c["hi"])])


def _requests(c):
    """Tokens that every request of a plan has cached, and those that it adds (-1: it has ended)."""
    lens, add = _spread(c["B"], c["lo"], c["hi"]), np.ones(c["B"], np.int64)
    if c["mixed"]:
        i = np.arange(c["B"])
        add[i % 8 == 3] = -1
        first = np.nonzero(i % 8 == 5)[0]
        lens[first] = 0
        add[first] = _spread(len(first), max(1, c["prompt"] // 16), c["prompt"])
    return lens, add


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))

    def on(a, dtype=torch.int32):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device=dev, dtype=dtype)

    def normal(*shape, sigma=1.0):
        # a page or a token at a time would be slow, a whole cache in 32 bits large: 64 M values at a time
        x = torch.empty(shape, dtype=_type(c), device=dev)
        for part in x.view(-1).split(1 << 26):
            part.copy_(torch.randn(part.shape, generator=gen, device=dev) * sigma)
        return x

    s = {"case": c}
    if c["kind"] == "plan":
        lens, add = _requests(c)
        order = rs.permutation(c["B"])
        lens, add, p = lens[order], add[order], c["page"]
        blocks = -(-lens // p)
        width = int((-(-(lens + np.maximum(add, 0)) // p)).max())
        total = int((-(-(lens + np.maximum(add, 0)) // p)).sum()) + 17
        pages = rs.permutation(total)
        table = np.full((c["B"], width), -1)
        table[np.arange(width)[None] < blocks[:, None]] = pages[:blocks.sum()]
        free = np.full(total, -1)
        free[:total - blocks.sum()] = pages[blocks.sum():]
        # the buffers are for 256 tokens at a time, as a program that captures its steps has them
        room = max(1, -(-int(np.maximum(add, 0).sum()) // 256)) * 256
        s.update(lens=on(lens), add=on(add), table=on(table), free=on(free), count=on([total - blocks.sum()]), page=p,
                 lens_new=on(np.zeros(c["B"])), cu=on(np.zeros(c["B"] + 1)), count_new=on([0]), status=on([0]),
                 positions=on(np.zeros(room)), slots=on(np.zeros(room), torch.int64))
        return s
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "attn":
        lens = rs.permutation(_lengths(c))
        p = c["page"]
        blocks = -(-lens // p)
        width, total = int(blocks.max()), int(blocks.sum()) + 5
        table = np.full((c["B"], width), -1)
        table[np.arange(width)[None] < blocks[:, None]] = rs.permutation(total)[:blocks.sum()]
        # a few keys stand out, as trained heads have them: scores of a deviation of two
        s["q"] = normal(c["B"], (Hq + 2 * Hkv) * D, sigma=2.0)[:, :Hq * D].unflatten(1, (Hq, D))
        s.update(k_cache=normal(total, Hkv, p, D), v_cache=normal(total, Hkv, p, D), table=on(table), lens=on(lens))
        s["out"] = torch.empty(c["B"], Hq, D, dtype=_type(c), device=dev)
        s["lse"] = torch.empty(c["B"], Hq, dtype=torch.float32, device=dev)
        return s
    n = c["tokens"]
    # queries, keys and values of one product, side by side
    qkv = normal(n, (Hq + 2 * Hkv) * D)
    s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
    s["wq"], s["wk"] = 1 + normal(D, sigma=0.2), 1 + normal(D, sigma=0.2)
    # whole sequences of positions where there is room, single far ones else
    pos = np.arange(n) % c["far"] if c["far"] <= n else np.sort(rs.randint(0, c["far"], n))
    s["pos"] = on(pos)
    s["freq"] = torch.from_numpy(10000.0 ** (-2.0 * np.arange(c["rot"] // 2) / c["rot"])).to(dev)
    s["q_out"], s["k_out"] = (torch.empty(n, h, D, dtype=_type(c), device=dev) for h in (Hq, Hkv))
    if c["kind"] == "bwd":
        s["dq_out"], s["dk_out"] = normal(n, Hq, D), normal(n, Hkv, D)
    if c["kind"] == "store":
        p = c["page"]
        total = -(-n // p) + 3
        s["slots"] = on(rs.permutation(total * p)[:n] if n < 256 else
                        (rs.permutation(total)[np.arange(n) // p] * p + np.arange(n) % p), torch.int64)
        s["k_cache"], s["v_cache"] = (torch.zeros(total, Hkv, p, D, dtype=_type(c), device=dev) for _ in range(2))
    return s


# ---------------------------------------------------------------- plain forms

def _plain_plan(s):
    p, table, free = s["page"], s["table"].long(), s["free"].long()
    lens, add, count = s["lens"].long(), s["add"].long(), s["count"].long()
    (B, W), F, room = table.shape, free.numel(), s["slots"].numel()
    dev = table.device
    ended, n = add < 0, add.clamp(min=0)
    old = (lens + p - 1) // p
    new_lens = torch.where(ended, 0, lens + n)
    new = (new_lens + p - 1) // p
    take, give = torch.where(ended, 0, new - old), torch.where(ended, old, 0)
    cu = torch.cat([torch.zeros_like(count), n.cumsum(0)])
    takes, gives = take.cumsum(0), give.cumsum(0)
    top = count + gives[-1]
    status = (cu[-1:] > room) * 1 + (new_lens.max() > W * p) * 2 + (takes[-1:] > top) * 4 + (top > F) * 8
    ok = status == 0
    # the stack of free pages with those that come back on top
    j = torch.arange(F, device=dev)
    r = (j - count).clamp(min=0)
    row = torch.searchsorted(gives, r, right=True).clamp(max=B - 1)
    back = table[row, (r - gives[row] + give[row]).clamp(0, W - 1)]
    stack = torch.where(j < count, free, back)
    left = top - takes[-1]
    free = torch.where(ok & (j >= count) & (j < left), stack, free)
    # pages that rows take, from its top down
    c = torch.arange(W, device=dev)[None]
    taken = ok & (c >= old[:, None]) & (c < (old + take)[:, None])
    index = top - 1 - ((takes - take - old)[:, None] + c)
    table = torch.where(taken, stack[index.clamp(0, F - 1)], table)
    t = torch.arange(room, device=dev)
    row = torch.searchsorted(cu[1:], t, right=True).clamp(max=B - 1)
    at = lens[row] + t - cu[row]
    valid = ok & (t < cu[-1])
    slots = torch.where(valid, table[row, (at // p).clamp(0, W - 1)] * p + at % p, -1)
    s["table"].copy_(table)
    s["free"].copy_(free)
    s["lens_new"].copy_(torch.where(ok, new_lens, lens))
    s["cu"].copy_(torch.where(ok, cu, 0))
    s["count_new"].copy_(torch.where(ok, left, count))
    s["status"].copy_(status)
    s["positions"].copy_(torch.where(valid, at, 0))
    s["slots"].copy_(slots)


def _angles(s):
    a = s["pos"].double()[:, None, None] * s["freq"]
    return a.cos().float(), a.sin().float()


def _turn(x, cos, sin, rot, pairs):
    """The first `rot` values of every head in pairs, each turned by its angle."""
    y = x.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


_EPS = 1e-6


def _plain_rope(s, x, w):
    c = s["case"]
    x, w = x.float(), w.float()
    x = x * (x.square().mean(-1, keepdim=True) + _EPS).rsqrt() * w
    return _turn(x, *_angles(s), c["rot"], c["pairs"]).to(_type(c))


def _plain_rope_bwd(s, x, w, dy):
    c = s["case"]
    x, w = x.float(), w.float()
    cos, sin = _angles(s)
    g = _turn(dy.float(), cos, -sin, c["rot"], c["pairs"])
    r = (x.square().mean(-1, keepdim=True) + _EPS).rsqrt()
    n = x * r
    gw = g * w
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx.to(_type(c)), (g * n).sum((0, 1))


def _plain_attn(s):
    c = s["case"]
    B, Hq, Hkv, D, p = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    table, lens = s["table"].long().clamp(min=0), s["lens"]
    L = table.shape[1] * p
    here = (torch.arange(L, device=lens.device) < lens[:, None])[:, None, :, None]

    def rows(cache):
        x = cache[table].transpose(1, 2).reshape(B, Hkv, L, D).float()
        return torch.where(here, x, 0.0)

    q = s["q"].float().reshape(B, Hkv, Hq // Hkv, D) * (1 / math.sqrt(D))
    z = torch.matmul(rows(s["k_cache"]), q.transpose(2, 3).contiguous())          # [B, Hkv, L, g]
    z = torch.where(here, z, float("-inf"))
    m = z.amax(2, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    e = torch.exp(z - m)
    l = e.sum(2, keepdim=True)
    o = torch.matmul(e.transpose(2, 3).contiguous(), rows(s["v_cache"]))
    o = o / torch.where(l == 0, 1.0, l).transpose(2, 3)
    return o.reshape(B, Hq, D).to(_type(c)), (m + torch.log(l)).reshape(B, Hq)


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "plan":
        return _plain_plan(s)
    if kind == "rope":
        return _plain_rope(s, s["q"], s["wq"]), _plain_rope(s, s["k"], s["wk"])
    if kind == "bwd":
        dq, dwq = _plain_rope_bwd(s, s["q"], s["wq"], s["dq_out"])
        dk, dwk = _plain_rope_bwd(s, s["k"], s["wk"], s["dk_out"])
        return dq, dk, dwq, dwk
    if kind == "store":
        c, p = s["case"], s["case"]["page"]
        page, off = s["slots"] // p, s["slots"] % p
        s["k_cache"][page, :, off] = _plain_rope(s, s["k"], s["wk"])
        s["v_cache"][page, :, off] = s["v"]
        return _plain_rope(s, s["q"], s["wq"])
    return _plain_attn(s)


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2405_03133_amd import binding as lb
    c = s["case"]
    kind = c["kind"]
    if kind == "plan":
        return lb.lory_kv_plan(s["lens"], s["add"], s["table"], s["free"], s["count"], s["page"], s["lens_new"], s["cu"],
                               s["positions"], s["slots"], s["count_new"], s["status"])
    if kind == "attn":
        if "ws" not in s:
            s["ws"] = lb.alloc_paged_attn_workspace(s["q"], s["k_cache"], s["table"])
        return lb.lory_paged_attn(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], out=s["out"], lse=s["lse"],
                                  workspace=s["ws"]), s["lse"]
    norm = dict(wq=s["wq"], wk=s["wk"], eps=_EPS, interleaved=c["pairs"])
    if kind == "rope":
        return lb.lory_qk_rope(s["q"], s["k"], s["pos"], s["freq"], q_out=s["q_out"], k_out=s["k_out"], **norm)
    if kind == "store":
        return lb.lory_qk_rope_cache(s["q"], s["k"], s["v"], s["pos"], s["freq"], s["k_cache"], s["v_cache"], s["slots"],
                                     q_out=s["q_out"], **norm)
    if "ws" not in s:
        s["ws"] = lb.alloc_qk_rope_workspace(s["q"], s["k"])
    return lb.lory_qk_rope_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], s["pos"], s["freq"], workspace=s["ws"], **norm)


def run(state):
    s = state
    kind = s["case"]["kind"]
    got = _own(s) if own else _plain(s)
    if kind == "plan":
        return {k: s[k] for k in ("table", "free", "count_new", "lens_new", "cu", "positions", "slots", "status")}
    if kind == "rope":
        return {"q": got[0], "k": got[1]}
    if kind == "bwd":
        return {"dq": got[0], "dk": got[1], "dwq": got[2], "dwk": got[3]}
    if kind == "store":
        return {"q": got, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return {"out": got[0], "lse": got[1]}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_rope(s, x, w):
    """x / sqrt(mean of squares) * w, its pairs as complex numbers times exp(i angle)."""
    c = s["case"]
    R = c["rot"]
    y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + _EPS) * w
    pair = y[..., :R].unflatten(-1, (R // 2, 2)) if c["pairs"] else y[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
    a = torch.outer(s["pos"].double(), s["freq"])[:, None, :]
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * torch.polar(torch.ones_like(a), a))
    z = z.flatten(-2) if c["pairs"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, y[..., R:]], -1)


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    c = case
    if c["kind"] == "attn":
        g, p = c["Hq"] // c["Hkv"], c["page"]
        out = torch.zeros(c["B"], c["Hq"], c["D"], dtype=torch.float64, device="cuda")
        lse = torch.full((c["B"], c["Hq"]), float("-inf"), dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["lens"].tolist()):
            if n == 0:
                continue
            pages = s["table"][b, :-(-n // p)].long()
            for h in range(c["Hkv"]):
                K, V = (x[pages, h].reshape(-1, c["D"])[:n].double() for x in (s["k_cache"], s["v_cache"]))
                z = s["q"][b, h * g:(h + 1) * g].double() @ K.T / math.sqrt(c["D"])
                out[b, h * g:(h + 1) * g] = torch.softmax(z, -1) @ V
                lse[b, h * g:(h + 1) * g] = torch.logsumexp(z, -1)
        return {"out": out, "lse": lse}
    q, k, wq, wk = (s[n].double().requires_grad_(c["kind"] == "bwd") for n in ("q", "k", "wq", "wk"))
    yq, yk = _exact_rope(s, q, wq), _exact_rope(s, k, wk)
    if c["kind"] == "rope":
        return {"q": yq, "k": yk}
    if c["kind"] == "bwd":
        got = torch.autograd.grad([yq, yk], [q, k, wq, wk], [s["dq_out"].double(), s["dk_out"].double()])
        return dict(zip(("dq", "dk", "dwq", "dwk"), got))
    K, V = (torch.zeros(s["k_cache"].shape, dtype=torch.float64, device="cuda").transpose(1, 2) for _ in range(2))
    K = K.reshape(-1, c["Hkv"], c["D"])
    V = V.reshape(-1, c["Hkv"], c["D"])
    K[s["slots"]], V[s["slots"]] = yk, s["v"].double()
    K, V = (x.unflatten(0, (-1, c["page"])).transpose(1, 2) for x in (K, V))
    return {"q": yq, "k_cache": K, "v_cache": V}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Every input read once, every output written once."""
    c = case
    if c["kind"] == "plan":
        lens, add = _requests(c)
        n, p = np.maximum(add, 0), c["page"]
        old, new = -(-lens // p), np.where(add < 0, 0, -(-(lens + n) // p))
        # lengths in and out with their offsets; a position and a slot a token; pages given back or taken are read and written
        moved = np.where(add < 0, old, new - old).sum()
        return {"bytes": int(4 * 4 * c["B"] + 12 * n.sum() + 8 * moved), "flops": int(10 * n.sum())}
    e = _esize(c)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "attn":
        n = int(_lengths(c).sum())
        blocks = int((-(-_lengths(c) // c["page"])).sum())
        return {"bytes": 2 * n * Hkv * D * e + c["B"] * Hq * (2 * D * e + 4) + 4 * blocks, "flops": 4 * n * Hq * D}
    n, values = c["tokens"], c["tokens"] * (Hq + Hkv) * D
    if c["kind"] == "rope":
        return {"bytes": 2 * values * e + 4 * n, "flops": 9 * values}
    if c["kind"] == "store":
        return {"bytes": 2 * (values + n * Hkv * D) * e + 12 * n, "flops": 9 * values}
    return {"bytes": 3 * values * e + 4 * n, "flops": 17 * values}
