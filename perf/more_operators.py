"""Several continuations of one prompt: what the operators of beam search and of parallel samples cost.

Four operators beside the plan and the paged attention of `operators.py`, as a program runs them that generates
several continuations of every request: the choice of the best continuations over beams and vocabulary, the
pages of a cache whose rows go on from other rows (shared, taken and given back), the copies of pages which that
asks for, and the attention of rows that have a long prefix in common.  Head counts are those of the widths that
`paper_2405_03133_amd.inputs.CONFIGS` has (1024, 1536, 2048, 4096) with heads of 64 or 128, some of them with
shared key-value heads; vocabularies and page sizes are generic.

`own` chooses between the plain forms below (elementary torch operations) and the calls of
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
        # one request of four beams after a step of a model with a small vocabulary: latency
        _case("select_b4", "select", dtype="bf16", R=1, K=4, k=8, V=32000, first=False),
        # a server's batch with a large vocabulary
        _case("select_batch", "select", dtype="bf16", R=48, K=8, k=16, V=128000, first=False),
        # the first step after the prompts, one live beam each; fp32 logits, rows that start at any address
        _case("select_first_odd", "select", dtype="f32", R=37, K=5, k=10, V=50257, first=True),
        # the prompts of a few requests become beams
        _case("fork_prompts", "fork", G=4, K=4, prompts=True, lo=100, hi=1500, grown=0, ended=0, page=16),
        # a step of a beam search over a batch: some beams end, others go on twice; some requests have ended
        _case("fork_beams", "fork", G=64, K=8, prompts=False, lo=300, hi=4000, grown=150, ended=7, page=16),
        # large pages, many samples of long prompts
        _case("fork_long", "fork", G=12, K=20, prompts=False, lo=5000, hi=100000, grown=3000, ended=2, page=64),
        # the last pages of one beam search step, partly filled, all layers of a cache in one call
        _case("copy_step", "copy", dtype="bf16", n=24, layers=4, Hkv=4, D=128, page=16, whole=False),
        # whole prefixes move
        _case("copy_prefix", "copy", dtype="bf16", n=3001, layers=1, Hkv=8, D=128, page=32, whole=True),
        # four beams of one request at the 0.3B width: latency
        _case("attn_b4", "attn", dtype="bf16", G=1, K=4, none=0, lo=1000, hi=1000, tail=40, Hq=16, Hkv=16, D=64, page=16),
        # a beam search over a batch at the headline width, shared heads, one request idle
        _case("attn_beams", "attn", dtype="bf16", G=24, K=8, none=1, lo=300, hi=6000, tail=150, Hq=16, Hkv=4, D=128, page=16),
        # one long prompt that a whole batch has in common, at the 4096 width
        _case("attn_system", "attn", dtype="bf16", G=1, K=96, none=0, lo=16000, hi=16000, tail=1500, Hq=32, Hkv=8, D=128, page=64),
        # fp32, groups of five heads of 80, three beams, pages that are no power of two
        _case("attn_f32_odd", "attn", dtype="f32", G=5, K=3, none=1, lo=3, hi=3001, tail=77, Hq=20, Hkv=4, D=80, page=24),
    ]


# ---------------------------------------------------------------- drawn cases

def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))))


def draw(rng):
    kind = rng.choice(["select", "fork", "copy", "attn", "attn"])
    while True:
        c = {"kind": kind}
        if kind == "select":
            c.update(dtype=rng.choice(["bf16", "bf16", "f32"]), R=_log(rng, 1, 200), K=rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 12, 16, 32]),
                     V=_log(rng, 900, 200000), first=rng.random() < 0.2)
            c["k"] = rng.choice([c["K"], 2 * c["K"], 2 * c["K"]])
            if rng.random() < 0.5:
                c["V"] = -(-c["V"] // 64) * 64
            if c["R"] * c["K"] * c["V"] * _esize(c) <= 48 * 8 * 128000 * 2:
                return c
            continue
        c["page"] = rng.choice([8, 16, 16, 24, 32, 64, 128])
        if kind == "fork":
            c.update(G=_log(rng, 1, 250), K=rng.choice([1, 2, 4, 4, 5, 8, 8, 16, 32]), prompts=rng.random() < 0.3, lo=_log(rng, 1, 2000))
            c["hi"] = c["lo"] + _log(rng, 1, 60000)
            c["grown"] = 0 if c["prompts"] else _log(rng, 1, 2000)
            c["ended"] = 0 if c["prompts"] else int(rng.random() * c["G"] / 3)
            if c["G"] * c["K"] * ((c["hi"] + c["grown"]) // c["page"] + 1) <= 500000:
                return c
            continue
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c["D"] = rng.choice([64, 128, 128, 128, 80, 96, 256])
        c["Hkv"] = rng.choice([1, 2, 4, 4, 8, 8, 16])
        if kind == "copy":
            c.update(n=_log(rng, 1, 4000), layers=rng.choice([1, 1, 2, 4, 24]), whole=rng.random() < 0.4)
            if c["n"] * c["layers"] * c["Hkv"] * c["page"] * c["D"] * _esize(c) <= 3001 * 8 * 32 * 128 * 2:
                return c
            continue
        c["Hq"] = c["Hkv"] * rng.choice([1, 2, 3, 4, 4, 5, 8] if c["Hkv"] <= 8 else [1, 2])
        c.update(G=_log(rng, 1, 60), K=_log(rng, 1, 100), hi=_log(rng, 1, 40000), tail=_log(rng, 1, 2000))
        c["lo"] = rng.choice([c["hi"], max(1, c["hi"] // 3), 1])
        c["none"] = rng.choice([0, 0, 1]) if c["G"] > 1 else 0
        if c["G"] * c["K"] * (c["hi"] + c["tail"]) * c["Hkv"] * c["D"] <= 96 * 17500 * 8 * 128 // 2:
            return c


# ---------------------------------------------------------------- inputs

def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _spread(n, lo, hi):
    """n lengths from lo to hi, even over their logarithm."""
    return np.rint(np.exp(np.linspace(math.log(lo), math.log(hi), n))).astype(np.int64) if n > 1 else np.array([hi] * n, np.int64)


def _ceil(a, b):
    return -(-a // b)


def _shared_table(prompt, lens, K, page, rs, spare, longest=0):
    """Page table of groups of K rows: whole pages of a group's prompt are shared, all others are each row's own."""
    G = len(prompt)
    used = _ceil(lens, page).reshape(G, K)
    W = max(1, int(used.max()), _ceil(longest, page))
    col = np.arange(W)[None, None]
    own_page = (col >= (prompt // page)[:, None, None]) & (col < used[:, :, None])
    common = (col < (prompt // page)[:, None, None]) & (col < used.max(1)[:, None, None])
    number = np.full((G, K, W), -1)
    n_common, n_own = int(common.sum()), int(own_page.sum())
    total = n_common + n_own + spare
    pages = rs.permutation(total)
    first = np.full((G, 1, W), -1)
    first[common] = pages[:n_common]
    number = np.where((col < used[:, :, None]) & ~own_page, first, number)
    number[own_page] = pages[n_common:n_common + n_own]
    return number.reshape(G * K, W), pages[n_common + n_own:], total


def _needed(prompt, lens, K, page):
    """Pages of such a table."""
    own_pages = _ceil(lens, page).reshape(-1, K) - (prompt // page)[:, None]
    return int((prompt // page).sum() + own_pages.sum())


def _group_lengths(c):
    """Prompts of an attention case's groups (0: idle) and the lengths of its rows."""
    G, K = c["G"], c["K"]
    prompt = np.concatenate([np.zeros(c["none"], np.int64), _spread(G - c["none"], c["lo"], c["hi"])])
    tail = 1 + (np.arange(G * K) * 7919) % c["tail"]
    return prompt, np.where(np.repeat(prompt, K) > 0, np.repeat(prompt, K) + tail, 0)


def _copy_rows(c):
    """Filled rows of the pages that are copied."""
    return np.full(c["n"], c["page"]) if c["whole"] else 1 + (np.arange(c["n"]) * 7919) % max(1, c["page"] - 1)


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))

    def on(a, dtype=torch.int32):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device=dev, dtype=dtype)

    def normal(*shape, sigma=1.0):
        # a page at a time would be slow, a whole cache in 32 bits large: 64 M values at a time
        x = torch.empty(shape, dtype=_type(c), device=dev)
        for part in x.view(-1).split(1 << 26):
            part.copy_(torch.randn(part.shape, generator=gen, device=dev) * sigma)
        return x

    s = {"case": c}
    if c["kind"] == "select":
        R, K, V, k = c["R"], c["K"], c["V"], c["k"]
        s["logits"] = normal(R * K, V, sigma=2.5)
        # tokens that may not follow, and beams that have ended
        barred = torch.rand(V, generator=gen, device=dev) < 0.01
        s["logits"].masked_fill_(barred, float("-inf"))
        score = -8 * torch.rand(R, K, generator=gen, device=dev).sort(1)[0] - 20
        ended = torch.rand(R, K, generator=gen, device=dev) < 0.05
        ended[:, 0] = False
        if c["first"]:
            ended[:, 1:] = True
        s["score"] = score.masked_fill(ended, float("-inf"))
        s["score_out"] = torch.empty(R, k, dtype=torch.float32, device=dev)
        s["token"], s["parent"] = (torch.empty(R, k, dtype=torch.int32, device=dev) for _ in range(2))
        return s
    p = c["page"]
    if c["kind"] == "fork":
        G, K = c["G"], c["K"]
        prompt = rs.permutation(_spread(G, c["lo"], c["hi"]))
        if c["prompts"]:
            lens = prompt
            table, free, total = _shared_table(prompt, lens, 1, p, rs, G * K + 23)
            src = np.repeat(np.arange(G), K)
        else:
            lens = np.repeat(prompt + rs.randint(0, c["grown"] + 1, G), K)
            # a pool of one size, whatever the lengths
            pool = int((prompt // p).sum()) + G * K * (_ceil(c["grown"], p) + 3) + 23
            table, free, total = _shared_table(prompt, lens, K, p, rs, pool - _needed(prompt, lens, K, p), c["hi"] + c["grown"])
            # better beams have more children
            best = np.minimum(rs.randint(0, K, (G, K)), rs.randint(0, K, (G, K)))
            src = (np.arange(G)[:, None] * K + np.sort(best, 1)).astype(np.int64)
            src[rs.permutation(G)[:c["ended"]]] = -1
            src = src.reshape(-1)
        stack = np.full(total, -1)
        stack[:len(free)] = free
        rows = len(src)
        s.update(lens=on(lens), src=on(src), table=on(table), free=on(stack), count=on([len(free)]), page=p, pages=total,
                 lens_new=on(np.zeros(rows)), table_new=on(np.full((rows, table.shape[1]), -1)), count_new=on([0]),
                 copies=on(np.zeros((3, rows))), status=on([0]))
        return s
    Hkv, D = c["Hkv"], c["D"]
    if c["kind"] == "copy":
        n = c["n"]
        total = 2 * n + n // 8 + 3
        s["k_cache"], s["v_cache"] = (normal(c["layers"], total, Hkv, p, D) for _ in range(2))
        order = rs.permutation(total)
        copies = np.stack([order[:n], order[n:2 * n], _copy_rows(c)])
        # most rows of a step copy nothing
        if not c["whole"]:
            full = np.stack([np.full(2 * n, -1), np.full(2 * n, -1), np.zeros(2 * n, np.int64)])
            full[:, np.sort(rs.permutation(2 * n)[:n])] = copies
            copies = full
        s["copies"] = on(copies)
        return s
    Hq, G, K = c["Hq"], c["G"], c["K"]
    prompt, lens = _group_lengths(c)
    order = rs.permutation(G)
    prompt, lens = prompt[order], lens.reshape(G, K)[order].reshape(-1)
    table, _, total = _shared_table(prompt, lens, K, p, rs, 5)
    s["k_cache"], s["v_cache"] = normal(total, Hkv, p, D), normal(total, Hkv, p, D)
    # the tokens of a prompt's last, partly filled page are in every row's own copy of it
    part = prompt % p
    page_of = table.reshape(G, K, -1)[np.arange(G), :, np.minimum(prompt // p, table.shape[1] - 1)]   # [G, K]
    g = np.nonzero((part > 0) & (prompt > 0))[0]
    if len(g) and K > 1:
        a, b = np.repeat(page_of[g, 0], K - 1), page_of[g, 1:].reshape(-1)
        for x in (s["k_cache"], s["v_cache"]):
            x[on(b, torch.int64)] = torch.where((torch.arange(p, device=dev) < on(np.repeat(part[g], K - 1))[:, None])[:, None, :, None],
                                                x[on(a, torch.int64)], x[on(b, torch.int64)])
    # a few keys stand out, as trained heads have them: scores of a deviation of two
    s["q"] = normal(G * K, (Hq + 2 * Hkv) * D, sigma=2.0)[:, :Hq * D].unflatten(1, (Hq, D))
    s.update(table=on(table), lens=on(lens), shared=on(prompt))
    s["out"] = torch.empty(G * K, Hq, D, dtype=_type(c), device=dev)
    s["lse"] = torch.empty(G * K, Hq, dtype=torch.float32, device=dev)
    return s


# ---------------------------------------------------------------- plain forms

def _plain_select(s):
    """score + log softmax, in 64 bits: neighbouring candidates of different beams may be near each other."""
    c = s["case"]
    R, K, V, k = c["R"], c["K"], c["V"], c["k"]
    x = s["logits"].double().view(R, K, V)
    m = x.amax(2, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    z = (x - (m + torch.log(torch.exp(x - m).sum(2, keepdim=True)))) + s["score"].double()[:, :, None]
    z = z.view(R, K * V)
    z = torch.where(torch.isnan(z), float("-inf"), z)
    # the k best; of those that equal the last, the ones with the lowest indices
    last = z.topk(min(k, K * V), 1)[0][:, -1:]
    above, tie = z > last, z == last
    room = k - above.sum(1, keepdim=True)
    taken = above | (tie & (tie.cumsum(1, dtype=torch.int32) <= room))
    index = torch.where(taken, torch.arange(K * V, device=z.device), K * V).topk(k, 1, largest=False)[0].sort(1)[0]
    value = torch.where(index < K * V, z.gather(1, index.clamp(max=K * V - 1)), float("-inf"))
    value, order = value.sort(dim=1, descending=True, stable=True)
    index = index.gather(1, order)
    none = value == float("-inf")
    beam = torch.arange(R, device=z.device)[:, None] * K + index // V
    s["score_out"].copy_(value)
    s["token"].copy_(torch.where(none, -1, index % V))
    s["parent"].copy_(torch.where(none, -1, beam))


def _plain_fork(s):
    p, pages = s["page"], s["pages"]
    lens, src, table, free, count = (s[n].long() for n in ("lens", "src", "table", "free", "count"))
    (B, W), N, F = table.shape, src.numel(), free.numel()
    dev = table.device
    live, parent = src >= 0, src.clamp(0, B - 1)
    row, col = torch.arange(N, device=dev), torch.arange(W, device=dev)
    used = (lens + p - 1) // p
    first = torch.full((B,), N, device=dev).scatter_reduce(0, parent, torch.where(live, row, N), "amin")
    length = torch.where(live, lens[parent], 0)
    part = length % p
    copy = live & (part > 0) & (first[parent] != row)
    # pages that some row goes on with, and those that only ended rows have
    inside = col < used[:, None]
    kept, old = (torch.zeros(pages + 1, dtype=torch.bool, device=dev) for _ in range(2))
    old[torch.where(inside, table, pages).view(-1)] = True
    kept[torch.where(inside & (first < N)[:, None], table, pages).view(-1)] = True
    back = (old & ~kept)[:pages]
    gives, takes = back.sum(), copy.sum()
    top = count + gives
    status = (takes > top) * 4 + (top > F) * 8 + ((src >= B).any() | (lens < 0).any() | (lens > W * p).any()) * 16
    ok = status == 0
    place = torch.where(back & ok, count + back.cumsum(0) - 1, F)
    stack = torch.cat([free, free[:1]]).scatter(0, place, torch.arange(pages, device=dev))[:F]
    left = top - takes
    j = torch.arange(F, device=dev)
    taken = stack[(top - copy.cumsum(0)).clamp(0, F - 1)]
    last = length // p
    new = torch.where(col < used[parent][:, None], table[parent], s["table_new"].long())
    new = torch.where(live[:, None], new, s["table_new"].long())
    new = torch.where(copy[:, None] & (col == last[:, None]), taken[:, None], new)
    s["table_new"].copy_(torch.where(ok, new, s["table_new"].long()))
    s["free"].copy_(torch.where(ok & (j >= count) & (j < left), stack, free))
    s["lens_new"].copy_(torch.where(ok, length, 0))
    s["count_new"].copy_(torch.where(ok, left, count))
    copy = copy & ok
    source = table[parent, last.clamp(max=W - 1)]
    s["copies"].copy_(torch.stack([torch.where(copy, source, -1), torch.where(copy, taken, -1), torch.where(copy, part, 0)]))
    s["status"].copy_(status)


def _plain_copy(s):
    copies = s["copies"].long()
    src, dst, rows = copies[:, copies[0] >= 0]
    here = (torch.arange(s["case"]["page"], device=src.device) < rows[:, None])[None, :, None, :, None]
    for x in (s["k_cache"], s["v_cache"]):
        x[:, dst] = torch.where(here, x[:, src], x[:, dst])


def _plain_attn(s):
    c = s["case"]
    B, Hq, Hkv, D, p = c["G"] * c["K"], c["Hq"], c["Hkv"], c["D"], c["page"]
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
    return {"select": _plain_select, "fork": _plain_fork, "copy": _plain_copy, "attn": _plain_attn}[kind](s)


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2405_03133_amd import binding as lb
    kind = s["case"]["kind"]
    if kind == "copy":
        return lb.lory_kv_copy(s["k_cache"], s["v_cache"], s["copies"])
    if kind == "select":
        if "ws" not in s:
            s["ws"] = lb.alloc_beam_select_workspace(s["logits"], s["score"], s["case"]["k"])
        return lb.lory_beam_select(s["logits"], s["score"], s["case"]["k"], score_out=s["score_out"], token=s["token"],
                                   parent=s["parent"], workspace=s["ws"])
    if kind == "fork":
        if "ws" not in s:
            s["ws"] = lb.alloc_kv_fork_workspace(s["src"], s["table"], s["pages"])
        return lb.lory_kv_fork(s["lens"], s["src"], s["table"], s["free"], s["count"], s["page"], s["pages"], s["lens_new"],
                               s["table_new"], s["count_new"], s["copies"], s["status"], workspace=s["ws"])
    if "ws" not in s:
        s["ws"] = lb.alloc_prefix_attn_workspace(s["q"], s["k_cache"], s["table"], s["shared"])
    return lb.lory_prefix_attn(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["shared"], out=s["out"],
                               lse=s["lse"], workspace=s["ws"]), s["lse"]


def run(state):
    s = state
    kind = s["case"]["kind"]
    got = _own(s) if own else _plain(s)
    names = {"select": ("score_out", "token", "parent"), "copy": ("k_cache", "v_cache"),
             "fork": ("table_new", "free", "count_new", "lens_new", "copies", "status")}
    if kind in names:
        return {n: s[n] for n in names[kind]}
    return {"out": got[0], "lse": got[1]}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c = case
    if c["kind"] == "fork":
        return None
    s = prepare(case, seed)
    if c["kind"] == "select":
        K, V, k = c["K"], c["V"], c["k"]
        out = {"score_out": [], "token": [], "parent": []}
        for r in range(c["R"]):
            z = torch.log_softmax(s["logits"][r * K:(r + 1) * K].double(), 1) + s["score"][r].double()[:, None]
            value, index = torch.sort(z.reshape(-1), descending=True, stable=True)
            value, index = value[:k], index[:k]
            none = value == float("-inf")
            out["score_out"].append(value)
            out["token"].append(torch.where(none, -1, index % V))
            out["parent"].append(torch.where(none, -1, r * K + index // V))
        return {n: torch.stack(x) for n, x in out.items()}
    if c["kind"] == "copy":
        K, V = s["k_cache"].double(), s["v_cache"].double()
        for a, b, n in zip(*s["copies"].tolist()):
            if a >= 0:
                K[:, b, :, :n], V[:, b, :, :n] = K[:, a, :, :n], V[:, a, :, :n]
        return {"k_cache": K, "v_cache": V}
    g, p, B = c["Hq"] // c["Hkv"], c["page"], c["G"] * c["K"]
    out = torch.zeros(B, c["Hq"], c["D"], dtype=torch.float64, device="cuda")
    lse = torch.full((B, c["Hq"]), float("-inf"), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, :_ceil(n, p)].long()
        for h in range(c["Hkv"]):
            K, V = (x[pages, h].reshape(-1, c["D"])[:n].double() for x in (s["k_cache"], s["v_cache"]))
            z = s["q"][b, h * g:(h + 1) * g].double() @ K.T / math.sqrt(c["D"])
            out[b, h * g:(h + 1) * g] = torch.softmax(z, -1) @ V
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Every input read once, every output written once; a prefix that rows share is one input."""
    c = case
    if c["kind"] == "select":
        n = c["R"] * c["K"] * c["V"]
        return {"bytes": n * _esize(c) + 4 * c["R"] * c["K"] + 12 * c["R"] * c["k"], "flops": 4 * n}
    if c["kind"] == "fork":
        # lengths, parents and copies; the table's entries in and out
        prompt = _spread(c["G"], c["lo"], c["hi"])
        entries = int(_ceil(prompt + c["grown"] // 2, c["page"]).sum())
        rows = c["G"] * c["K"]
        old = entries if c["prompts"] else entries * c["K"]
        return {"bytes": 4 * (old + entries * c["K"]) + 24 * rows, "flops": entries * c["K"]}
    if c["kind"] == "copy":
        return {"bytes": int(4 * _copy_rows(c).sum()) * c["layers"] * c["Hkv"] * c["D"] * _esize(c) + 12 * c["n"], "flops": 0}
    prompt, lens = _group_lengths(c)
    e, Hq, Hkv, D, B = _esize(c), c["Hq"], c["Hkv"], c["D"], c["G"] * c["K"]
    tokens = int(prompt.sum() + (lens - np.repeat(prompt, c["K"])).sum())
    return {"bytes": 2 * tokens * Hkv * D * e + B * Hq * (2 * D * e + 4) + 4 * B * 2, "flops": 4 * int(lens.sum()) * Hq * D}
