"""Several continuations of one prompt (selection, forked rows of the cache, copies of pages, a shared prefix) against plain
implementations in 64 bits or in whole numbers.

Bounds are counted, not measured, as in test_attn_gpu.py; the multiples of 2^-24 are at each check."""
import numpy as np
import pytest
import torch

from paper_2405_03133_amd import binding as lb
from test_attn_gpu import E32, T, check_attention, gen, paged_case, rnd, same, within

pytestmark = pytest.mark.gpu

NONE = float("-inf")


def i32(a):
    return torch.from_numpy(np.asarray(a).copy()).to(dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- selection

def select(logits, score, k):
    ws = lb.alloc_beam_select_workspace(logits, score, k)
    ws.fill_(255)
    out = lb.lory_beam_select(logits, score, k, workspace=ws)
    ws.fill_(1)
    again = lb.lory_beam_select(logits, score, k, workspace=ws)
    own = lb.lory_beam_select(logits, score, k)
    for a, b, c in zip(out, again, own):
        assert torch.equal(a, b) and torch.equal(a, c)
    return out


def check_select(label, logits, score, k, out=None):
    """The choice within a beam is that of the logits, exactly; between beams it may differ where candidates are nearer each
    other than the sums of exponentials are accurate."""
    R, K = score.shape
    V = logits.shape[1]
    got_score, token, parent = out or select(logits, score, k)
    x = logits.double().view(R, K, V)
    odd = (torch.isnan(x) | (x == float("inf"))).any(2, keepdim=True)
    x = torch.where(odd, NONE, x)
    lse = torch.logsumexp(x, 2, keepdim=True)
    lse = torch.where(lse == NONE, 0.0, lse)
    # a term: the argument's two roundings and the constant's (3 of its size), the exponential (2); a lane's chain of 64 additions;
    # the sums over lanes are in 64 bits
    top = x.amax(2, keepdim=True)
    top = torch.where(top == NONE, 0.0, top)
    p = torch.exp(x - lse)
    far = (p * (top - x).clamp(max=1000).nan_to_num(0.0)).sum(2)
    dl = ((3 * far + 66) * E32).amax(1)                                     # [R]
    z = x - lse + score.double()[:, :, None]
    z = torch.where(torch.isnan(z), NONE, z).view(R, K * V)
    ref, index = z.sort(dim=1, descending=True, stable=True)
    n = min(k, K * V)
    ref, index = ref[:, :n], index[:, :n]
    # what is no candidate
    assert token.shape == parent.shape == got_score.shape == (R, k)
    count = (ref > NONE).sum(1, keepdim=True)
    there = torch.arange(k, device="cuda") < count
    assert (got_score[~there] == NONE).all() and (token[~there] == -1).all() and (parent[~there] == -1).all(), label
    assert (token[there] >= 0).all() and (token[there] < V).all() and (got_score[there] > NONE).all(), label
    beam = parent.long() - torch.arange(R, device="cuda")[:, None] * K
    assert (beam[there] >= 0).all() and (beam[there] < K).all(), label
    there = there[:, :n]
    got = (beam * V + token)[:, :n]
    got = torch.where(there, got, index)
    value = z.gather(1, got)
    # the same candidates but for near ones, in order, each once
    assert (torch.where(there, (value - ref).abs() <= 2 * dl[:, None], True) | (value == ref)).all(), label
    same_beam = (got == index) | ~there
    for r in range(R):
        if same_beam[r].all():
            continue
        for b in range(K):   # of each beam its first ones
            mine = got[r][there[r] & (got[r] // V == b)] - b * V
            first = x[r, b].sort(descending=True, stable=True)[1][:mine.numel()]
            assert torch.equal(mine, first), (label, r, b)
    within(f"{label} score", got_score[:, :n][there], value[there], dl[:, None].expand(R, n)[there], torch.float32)
    s = got_score[:, :n]
    assert (s[:, 1:] <= s[:, :-1]).all(), label
    print(f"[beam] {label}: {(~same_beam).sum().item()} of {same_beam.numel()} in another order", flush=True)


def logits_of(g, rows, V, dtype, sigma=2.5):
    return (rnd(g, rows, V) * sigma).to(T[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,K,V,k", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 1, 4), (3, 4, 1000, 8), (2, 3, 50257, 6), (1, 64, 300, 64),
                                     (5, 2, 131072, 4), (2, 5, 33001, 10), (1, 1, 500000, 64), (7, 16, 4097, 32), (300, 1, 2000, 1),
                                     (1, 64, 499999, 64), (40, 8, 32000, 16), (1, 2, 8191, 3)])
def test_select(R, K, V, k, dtype):
    g = gen(R + V)
    score = -20 * torch.rand(R, K, generator=g, device="cuda")
    check_select(f"{R}x{K}x{V} k {k}", logits_of(g, R * K, V, dtype), score, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1, 3, 5])
def test_select_rows_anywhere(off, dtype):
    """Rows that start at any address of their type, with neighbours that would win."""
    g = gen(off)
    V = 9001
    wide = torch.full((12, V + 37), 1000.0, device="cuda", dtype=T[dtype])
    x = wide[:, off:off + V]
    x.copy_(logits_of(g, 12, V, dtype))
    score = -torch.rand(4, 3, generator=g, device="cuda")
    a = select(x, score, 6)
    check_select("slice", x, score, 6, a)
    for i, j in zip(a, select(x.contiguous(), score, 6)):
        assert torch.equal(i, j)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_equal_logits(dtype):
    """Equal candidates: by beam, then by token; thousands of them, and a few distinct values."""
    R, K, V = 2, 3, 70000
    score = torch.zeros(R, K, device="cuda")
    for k in (1, 7, 64):
        _, token, parent = select(torch.zeros(R * K, V, device="cuda", dtype=T[dtype]), score, k)
        assert (token == torch.arange(k, device="cuda")).all() and (parent == torch.tensor([[0], [K]], device="cuda")).all()
    g = gen(1)
    x = torch.randint(0, 3, (R * K, V), generator=g, device="cuda").to(T[dtype])
    x[:, ::2] *= -1.0                                        # zeros of both signs are equal
    check_select("three values", x, score, 20)
    x = torch.randint(0, 2, (R * K, V), generator=g, device="cuda").to(T[dtype])
    check_select("two values", x - 100, score, 64)
    # identical beams: the lower one first
    x = logits_of(g, 1, 5000, dtype).expand(4, 5000).contiguous()
    _, token, parent = select(x, torch.full((1, 4), -3.0, device="cuda"), 8)
    assert parent[0].tolist() == [0, 1, 2, 3] * 2 and token[0, 0] == token[0, 3] and token[0, 4] == token[0, 7]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 40000])
def test_select_what_is_no_candidate(V, dtype):
    g = gen(V)
    R, K, k = 8, 4, 8
    x, score = logits_of(g, R * K, V, dtype), -torch.rand(R, K, generator=g, device="cuda")
    score[0, 1:] = NONE                                      # one live beam
    score[1] = NONE                                          # none
    x[8:12] = NONE                                           # request 2: nothing may follow
    x[12:16, 3:] = NONE                                      # request 3: three tokens
    x[12, :3] = NONE                                         # and none of its first beam
    x[16, V // 2] = float("nan")                             # request 4: a beam without a distribution
    x[20, V - 1] = float("inf")
    x[24:28] = torch.where(torch.arange(V, device="cuda") % 17 == 0, x[24:28], NONE)
    score[7, 2] = float("nan")
    x[28:32] = torch.finfo(T[dtype]).min                     # the lowest value, all alike
    check_select("odd", x, score, k)
    s, token, parent = select(x, score, k)
    assert (parent[4] != 16).all() and (parent[5] != 20).all() and (parent[7] != 30).all() and (parent[3] != 12).all()
    assert (token[1] == -1).all() and (token[2] == -1).all() and (parent[0] == 0).all() and (s[7] > NONE).all()


def test_select_large_logits_and_far_scores():
    g = gen(5)
    x = logits_of(g, 6, 3000, "f32", sigma=1e4)
    score = torch.tensor([[0.0, -1e6, 1e6], [-1e30, -1e30, -3e38]], device="cuda")
    check_select("large", x, score, 12)
    x[:, 0] = torch.finfo(torch.float32).max
    x[:, 1] = -torch.finfo(torch.float32).max
    check_select("to the ends", x, score, 12)


def test_select_many_rows():
    g = gen(6)
    x, score = logits_of(g, 70000, 64, "bf16"), torch.zeros(70000, 1, device="cuda")
    s, token, parent = select(x, score, 2)
    value, index = x.float().sort(dim=1, descending=True, stable=True)
    assert torch.equal(token.long(), index[:, :2]) and torch.equal(parent, i32(np.arange(70000))[:, None].expand(-1, 2))
    within("many", s, torch.log_softmax(x.double(), 1).gather(1, index[:, :2]), torch.full((70000, 2), 200 * E32, device="cuda"),
           torch.float32)


# ---------------------------------------------------------------- forked rows

def fork_oracle(lens, src, table, free, count, page, pages):
    """Python integers only."""
    B, W, F, N = len(lens), len(table[0]) if len(table) else 0, len(free), len(src)
    used = lambda n: -(-n // page)
    status = 0
    if not 0 <= count <= F or any(s >= B for s in src) or any(not 0 <= n <= W * page for n in lens):
        status = 16
    elif any(not 0 <= table[b][c] < pages for b in range(B) for c in range(used(lens[b]))):
        status = 16
    if status:
        return status, None
    old = {table[b][c] for b in range(B) for c in range(used(lens[b]))}
    kept = {table[s][c] for s in src if s >= 0 for c in range(used(lens[s]))}
    stack = free[:count] + sorted(old - kept)
    seen, takers = set(), []
    for b, s in enumerate(src):
        if s >= 0:
            if lens[s] % page and s in seen:
                takers.append(b)
            seen.add(s)
    if len(takers) > len(stack):
        status |= 4
    if len(stack) > F:
        status |= 8
    if status:
        return status, None
    new, copies = [None] * N, [[-1] * N, [-1] * N, [0] * N]
    for b, s in enumerate(src):
        new[b] = list(table[s][:used(lens[s])]) if s >= 0 else []
    for b in takers:
        n = lens[src[b]]
        to = stack.pop()
        copies[0][b], copies[1][b], copies[2][b] = new[b][-1], to, n % page
        new[b][-1] = to
    return 0, (new, stack, [lens[s] if s >= 0 else 0 for s in src], copies)


def run_fork(lens, src, table, free, count, page, pages, wide=0):
    B, N, W = len(lens), len(src), len(table[0])
    tall = i32(np.full((max(B, 1), W + wide), -9))
    tall[:B, :W] = i32(np.asarray(table).reshape(-1, W)[:B])
    new = i32(np.full((max(N, 1), W + 2 * wide), -5))
    s = dict(lens=i32(lens), src=i32(src), table=tall[:B, :W], free=i32(free), count=i32([count]), lens_new=i32([77] * N),
             table_new=new[:N, :W], count_new=i32([77]), copies=i32(np.full((3, N), 77)), status=i32([77]))
    ws = lb.alloc_kv_fork_workspace(s["src"], s["table"], pages)
    ws.fill_(255)
    call = lambda **kw: lb.lory_kv_fork(s["lens"], s["src"], s["table"], s["free"], s["count"], page, pages, s["lens_new"], s["table_new"],
                                        s["count_new"], s["copies"], s["status"], **kw)
    call(workspace=ws)
    first = {n: x.clone() for n, x in s.items()}
    call()
    for n, x in s.items():
        assert torch.equal(x, first[n]), n            # the same again
    assert (new[:N, W:] == -5).all() and torch.equal(s["table"], i32(np.asarray(table).reshape(-1, W)[:B]))
    return {n: x.cpu().numpy() for n, x in s.items()}


def check_fork(lens, src, table, free, count, page, pages, wide=0):
    got = run_fork(lens, src, table, free, count, page, pages, wide)
    status, want = fork_oracle(list(map(int, lens)), list(map(int, src)), [list(map(int, r)) for r in table], list(map(int, free)),
                               int(count), page, pages)
    assert got["status"][0] == status, (got["status"], status)
    N = len(src)
    if status:
        assert (got["free"] == np.asarray(free)).all() and got["count_new"][0] == count and (got["lens_new"] == 0).all()
        assert (got["copies"][:2] == -1).all() and (got["copies"][2] == 0).all()
        return got
    new, stack, lens_new, copies = want
    assert got["count_new"][0] == len(stack)
    assert got["free"][:len(stack)].tolist() == stack
    assert (got["free"][max(count, len(stack)):] == np.asarray(free)[max(count, len(stack)):]).all()      # nothing above is written
    assert got["lens_new"].tolist() == lens_new and got["copies"].tolist() == copies
    for b in range(N):
        n = len(new[b])
        assert got["table_new"][b, :n].tolist() == new[b], b
        assert (got["table_new"][b, n:] == -5).all(), b
    return got


def fork_state(rs, G, K, page, hi, extra=0):
    """Requests of K rows each, their prompts' whole pages shared."""
    prompt = rs.randint(0, hi, G)
    lens = np.repeat(prompt, K) + rs.randint(0, 3 * page, G * K)
    used = -(-lens // page)
    W = int(used.max()) + 1
    total = int(used.sum()) + G * K + extra + 1
    perm = rs.permutation(total).tolist()
    table = rs.choice([-1, 2 ** 31 - 1, total], size=(G * K, W))
    for g in range(G):
        common = [perm.pop() for _ in range(prompt[g] // page)]
        for r in range(g * K, (g + 1) * K):
            own = [perm.pop() for _ in range(used[r] - len(common))]
            table[r, :used[r]] = common + own
    free = np.full(total, -1)
    free[:len(perm)] = perm
    return lens, table, free, len(perm), total


@pytest.mark.parametrize("G,K,page,hi", [(1, 1, 16, 40), (1, 4, 16, 100), (3, 5, 1, 30), (7, 8, 24, 300), (60, 8, 16, 900), (2, 33, 128, 5000),
                                         (300, 2, 8, 50), (1, 1500, 16, 200), (12, 20, 64, 20000)])
def test_fork(G, K, page, hi):
    rs = np.random.RandomState(G * K + page)
    lens, table, free, count, pages = fork_state(rs, G, K, page, hi)
    B = G * K
    n = np.arange(B)
    sources = [(n // K) * K + np.sort(np.minimum(rs.randint(0, K, (G, K)), rs.randint(0, K, (G, K))), 1).reshape(-1),   # a beam step
               n, n[::-1], np.full(B, -1), np.where(rs.rand(B) < 0.4, -1, rs.permutation(B)), np.zeros(B, int), rs.randint(-1, B, B),
               rs.randint(-1, B, 3 * B + 1), rs.randint(-1, B, max(1, B // 3)), np.zeros(0, int)]
    for i, src in enumerate(sources):
        check_fork(lens, src, table, free, count, page, pages, wide=i % 3)


def test_fork_of_prompts_takes_pages_that_come_back():
    """An empty stack: the pages that copies need are those of a row that ends."""
    table = [[3, 1, -1], [0, 4, 2]]
    got = check_fork([24, 40], [0, 0, 0], table, [-1] * 5, 0, 16, 5)
    assert got["copies"].tolist() == [[-1, 1, 1], [-1, 4, 2], [0, 8, 8]] and got["count_new"][0] == 1 and got["free"][0] == 0
    got = check_fork([24, 40], [0, 0, 0, 0, 0], table, [-1] * 5, 0, 16, 5)
    assert got["status"][0] == 4
    # rows of whole pages share all of them
    got = check_fork([32, 0], [0, 0, 1, 0], table, [-1] * 5, 0, 16, 5)
    assert (got["copies"][0] == -1).all() and got["table_new"][:2, :2].tolist() == [[3, 1]] * 2


@pytest.mark.parametrize("change,status", [(dict(count=6), 8), (dict(count=9), 16), (dict(count=-1), 16), (dict(lens=[-1, 40]), 16),
                                           (dict(lens=[24, 49]), 16), (dict(src=[0, 2]), 16), (dict(src=[0, 2 ** 31 - 1]), 16),
                                           (dict(table=[[3, 7, -1], [0, 4, 2]]), 16), (dict(table=[[3, -1, -1], [0, 4, 2]]), 16),
                                           (dict(table=[[3, 1, 9], [0, 4, -2 ** 31]]), 16)])
def test_fork_status(change, status):
    a = dict(lens=[24, 40], src=[0, 0], table=[[3, 1, -1], [0, 4, 2]], free=[5, 6, -1, -1, -1, -1, -1, -1], count=2, page=16, pages=7)
    assert check_fork(**a)["status"][0] == 0
    a.update(change)
    assert check_fork(**a)["status"][0] == status


def test_fork_of_a_large_pool():
    """Tables of half a million entries over a pool of a million pages."""
    rs = np.random.RandomState(3)
    B, W, page, pages = 512, 1000, 16, 1 << 20
    lens = rs.randint(0, W * page + 1, B)
    lens[:8] = W * page
    table = rs.permutation(pages)[:B * W].reshape(B, W)
    table[100:200, :300] = table[99, :300]
    free = np.full(pages, -1)
    free[:700] = np.arange(700)
    check_fork(lens, np.sort(rs.randint(-1, B, 700)), table, free, 700, page, pages)


def test_fork_of_nothing():
    got = check_fork([16, 5], [], [[1], [0]], [-1] * 4, 0, 16, 2)
    assert got["free"][:2].tolist() == [0, 1] and got["count_new"][0] == 2
    s = [i32([]), i32([-1, -3]), torch.zeros(0, 4, dtype=torch.int32, device="cuda"), i32([5]), i32([1])]
    out = [i32([7, 7]), i32(np.zeros((2, 4))), i32([0]), i32(np.zeros((3, 2))), i32([5])]
    lb.lory_kv_fork(*s, 16, 8, *out)
    assert out[0].tolist() == [0, 0] and out[2].item() == 1 and out[3].tolist() == [[-1, -1], [-1, -1], [0, 0]] and out[4].item() == 0


# ---------------------------------------------------------------- copies

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layers,pages,Hkv,page,D", [(0, 9, 1, 1, 8), (0, 40, 3, 16, 64), (3, 30, 4, 24, 80), (2, 25, 2, 128, 256), (24, 12, 1, 8, 128)])
def test_copy(layers, pages, Hkv, page, D, dtype):
    g = gen(pages)
    rs = np.random.RandomState(pages)
    shape = (layers, pages, Hkv, page, D) if layers else (pages, Hkv, page, D)
    k, v = rnd(g, *shape, dtype=T[dtype]), rnd(g, *shape, dtype=T[dtype])
    k.view(-1)[5], v.view(-1)[7] = float("nan"), float("inf")
    order = rs.permutation(pages)
    n = pages // 3
    copies = np.stack([order[:n], order[n:2 * n], rs.randint(1, page + 1, n)])
    copies[0, 1:] = np.where(rs.rand(n - 1) < 0.3, copies[0, 0], copies[0, 1:])      # one page to several
    odd = np.array([[-1, 0, pages, 3, order[0], 2 ** 31 - 1, order[1], order[2]], [0, -1, 1, pages, order[-1], -2 ** 31, order[1], order[-2]],
                    [page, page, page, page, 0, page, page, -4]])                     # pairs that copy nothing
    copies = np.concatenate([copies, odd, [[order[0]], [order[-3]], [page + 100]]], 1)   # more than a page: a page
    wk, wv = k.clone(), v.clone()
    d = 1 if layers else 0
    for a, b, m in copies.T.tolist():
        if 0 <= a < pages and 0 <= b < pages and a != b and m > 0:
            for x, w in ((k, wk), (v, wv)):
                w.select(d, b)[..., :m, :] = x.select(d, a)[..., :m, :]
    lb.lory_kv_copy(k, v, i32(copies))
    assert same(k, wk) and same(v, wv)
    lb.lory_kv_copy(k, v, i32(np.zeros((3, 0))))
    assert same(k, wk)


def test_copy_above_32_bits():
    Hkv, page, D = 2, 64, 128
    per = Hkv * page * D * 2
    pages = (1 << 33) // per + 70
    k, v = (torch.empty(pages, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    g = gen(2)
    src = [0, (1 << 32) // per, pages - 1]
    dst = [(1 << 33) // per, 5, (1 << 31) // per]
    for i in src + dst:
        k[i], v[i] = rnd(g, Hkv, page, D).bfloat16(), rnd(g, Hkv, page, D).bfloat16()
    lb.lory_kv_copy(k, v, i32([src, dst, [page, page, page - 1]]))
    for a, b, m in zip(src, dst, (page, page, page - 1)):
        assert torch.equal(k[b, :, :m], k[a, :, :m]) and torch.equal(v[b, :, :m], v[a, :, :m])
    assert not torch.equal(k[dst[2], :, -1], k[src[2], :, -1])


def test_copy_of_many_pairs():
    k, v = (torch.randn(140010, 1, 1, 8, device="cuda") for _ in range(2))
    n = 70000
    want = k[:n].clone()
    copies = torch.stack([torch.arange(n), torch.arange(n) + n, torch.ones(n, dtype=torch.long)]).int().cuda()
    lb.lory_kv_copy(k, v, copies)
    assert torch.equal(k[n:2 * n], want) and torch.equal(v[n:2 * n], v[:n])


# ---------------------------------------------------------------- a prefix that rows share

def prefix_case(seed, prefix, tails, Hq, Hkv, D, page, dtype, **kw):
    """Groups with prefixes of these lengths; tails[g]: lengths behind it of its rows, None: an idle row, below 0: a shorter row.  Rows of
    a group share the prefix's whole pages, and have copies of the last one."""
    K = len(tails[0])
    lens = [0 if t is None else max(0, p + t) for p, ts in zip(prefix, tails) for t in ts]
    q, k, v, table, dlens = paged_case(seed, lens, Hq, Hkv, D, page, dtype, **kw)
    tab = table.cpu().numpy()
    for g, p in enumerate(prefix):
        rows = [b for b in range(g * K, (g + 1) * K) if lens[b] >= p > 0]
        for b in rows[1:]:
            tab[b, :p // page] = tab[rows[0], :p // page]
            part = p % page
            if part:
                a, c = tab[rows[0], p // page], tab[b, p // page]
                k[c, :, :part], v[c, :, :part] = k[a, :, :part], v[a, :, :part]
    return (q, k, v, i32(tab), dlens), i32(prefix)


def prefixed(case, shared, **kw):
    q, k, v, table, lens = case
    lse = torch.full(q.shape[:2], 77.0, device="cuda")
    ws = lb.alloc_prefix_attn_workspace(q, k, table, shared)
    ws.fill_(255)
    out = lb.lory_prefix_attn(q, k, v, table, lens, shared, lse=lse, workspace=ws, **kw)
    lse2 = torch.empty_like(lse)
    assert same(out, lb.lory_prefix_attn(q, k, v, table, lens, shared, lse=lse2, **kw)) and same(lse, lse2)
    assert same(out, lb.lory_prefix_attn(q, k, v, table, lens, shared, **kw))   # without lse
    return out, lse


PREFIX = [0, 1, 15, 16, 17, 31, 32, 63, 65, 127, 128, 129, 500, 1000, 7, 40]


def tails_of(rs, G, K, hi):
    t = rs.randint(0, hi, (G, K)).tolist()
    t[G - 1] = [None] * K                     # an idle group
    if K > 1:
        t[0][0] = None
        t[2][K - 1] = None
        t[4][0], t[5][K // 2] = -3, -31       # rows that have only a part of it, or none
        t[12] = [-1] * K                      # a group of which no row has all of it
    return t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,Hq,Hkv,D,page", [(1, 4, 2, 64, 16), (4, 16, 16, 64, 16), (3, 20, 4, 80, 24), (5, 8, 1, 128, 16), (8, 16, 4, 128, 32),
                                             (2, 40, 1, 128, 64), (7, 6, 2, 256, 8), (33, 2, 1, 64, 16), (20, 8, 2, 128, 16), (9, 4, 4, 8, 1),
                                             (16, 3, 1, 200, 24)])
def test_prefix_attention(K, Hq, Hkv, D, page, dtype):
    rs = np.random.RandomState(K + D)
    case, shared = prefix_case(K + Hq, PREFIX, tails_of(rs, len(PREFIX), K, 90), Hq, Hkv, D, page, dtype)
    check_attention(f"prefix {K} rows {Hq}/{Hkv}x{D}", *prefixed(case, shared), *case)


@pytest.mark.parametrize("prefix,K,tail,Hq,Hkv,D,page,dtype", [
    ([9000], 4, 300, 8, 2, 128, 16, "bf16"), ([20000, 1, 5000], 6, 2000, 8, 8, 64, 64, "bf16"), ([3001, 0, 40], 3, 2500, 20, 4, 80, 24, "f32"),
    ([6000], 40, 50, 8, 2, 128, 16, "bf16"), ([4000, 4000], 16, 9, 16, 1, 128, 128, "bf16"), ([5000], 20, 700, 4, 2, 256, 16, "f32"),
    ([2000] * 30, 2, 100, 4, 2, 64, 16, "bf16"), ([1, 2, 3], 50, 600, 4, 1, 128, 16, "bf16"), ([8000], 1, 4000, 6, 2, 96, 32, "f32")])
def test_prefix_attention_split_over_the_cache(prefix, K, tail, Hq, Hkv, D, page, dtype):
    rs = np.random.RandomState(K)
    tails = rs.randint(0, tail, (len(prefix), K)).tolist()
    case, shared = prefix_case(3, prefix, tails, Hq, Hkv, D, page, dtype)
    check_attention(f"prefix {prefix[:2]} {K} rows", *prefixed(case, shared), *case)


@pytest.mark.parametrize("K,Hq,Hkv,D,dtype", [(4, 8, 2, 128, "bf16"), (12, 8, 2, 64, "bf16"), (3, 4, 2, 128, "f32")])
def test_prefix_attention_of_a_large_cache(K, Hq, Hkv, D, dtype):
    """Large caches are read another way."""
    rs = np.random.RandomState(1)
    case, shared = prefix_case(5, [700, 0, 3000], rs.randint(0, 500, (3, K)).tolist(), Hq, Hkv, D, 16, dtype, least_bytes=70 << 20)
    check_attention(f"large cache {K} rows", *prefixed(case, shared), *case)


def test_prefix_attention_of_many_rows():
    """Groups of one row and a prefix of nothing are the plain attention; 70000 rows pass a grid dimension."""
    B, D, page = 70000, 8, 4
    g = gen(3)
    lens = torch.randint(0, 5, (B,), generator=g, device="cuda", dtype=torch.int32)
    k, v = rnd(g, 1000, 1, page, D), rnd(g, 1000, 1, page, D)
    table = torch.randint(0, 1000, (B, 1), generator=g, device="cuda", dtype=torch.int32)
    q = rnd(g, B, 1, D)
    want = lb.lory_paged_attn(q, k, v, table, lens)
    for groups in (B, B // 7):
        shared = torch.zeros(groups, dtype=torch.int32, device="cuda")
        out = lb.lory_prefix_attn(q, k, v, table, lens, shared)
        # both have a chain of at most 70 additions on values that are averages of these
        within("many", out, want.double(), torch.full_like(want, 200 * E32 * float(v.abs().max())).double(), torch.float32)


def test_prefix_attention_strides_scale_and_in_place():
    Hq, Hkv, D, page = 6, 2, 128, 16
    case, shared = prefix_case(2, [40, 300], [[5, 0, None], [1, 70, 33]], Hq, Hkv, D, page, "bf16")
    q, k, v, table, lens = case
    wide = torch.full((6, (Hq + 4) * D), 5.0, device="cuda", dtype=torch.bfloat16)
    qs = wide[:, :Hq * D].unflatten(1, (Hq, D))
    qs.copy_(q)
    tall = torch.full((6, table.shape[1] + 9), -7, device="cuda", dtype=torch.int32)
    tall[:, :table.shape[1]] = table
    view = tall[:, :table.shape[1]]
    want, lse = prefixed(case, shared, scale=0.3)
    check_attention("scale", want, lse, *case, scale=0.3)
    outside = torch.empty(Hq, 6, D, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    assert torch.equal(lb.lory_prefix_attn(qs, k, v, view, lens, shared, out=outside, scale=0.3), want)
    assert lb.lory_prefix_attn(qs, k, v, view, lens, shared, out=qs, scale=0.3) is qs and torch.equal(qs, want)
    assert (wide[:, Hq * D:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_attention_bounds(dtype):
    """Lengths and prefixes below 0 and above the table; pages that are none."""
    case, shared = prefix_case(4, [48, 20], [[0, 0], [28, 12]], 2, 2, 64, 16, dtype)
    q, k, v, table, _ = case
    dev = lambda *a: torch.tensor(a, device="cuda", dtype=torch.int32)
    for lens, sh, count in [((2 ** 31 - 1, 48, -5, 20), (2 ** 31 - 1, 20), (48, 48, 0, 20)), ((48, 40, 48, 20), (48, -7), (48, 40, 48, 20)),
                            ((48, 47, 3, 2), (2 ** 31 - 1, -2 ** 31), (48, 47, 3, 2)), ((0, 0, 0, 0), (5, 0), (0, 0, 0, 0))]:
        out, lse = prefixed((q, k, v, table, dev(*lens)), dev(*sh))
        check_attention(f"bounds {lens}", out, lse, q, k, v, table, dev(*count))
    table = table.clone()
    table[:2, 1], table[2, 0], table[3, 0] = -1, k.shape[0], 2 ** 31 - 1
    case = (q, k, v, table, dev(48, 48, 48, 20))
    check_attention("no pages", *prefixed(case, shared), *case, skip={0: range(16, 32), 1: range(16, 32), 2: range(16), 3: range(16)})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 3, 20])
def test_prefix_attention_extreme_scores(K, dtype):
    """-inf scores, lowest values, large scores; NaN and infinities stay in their heads and rows."""
    t = T[dtype]
    tails = [[5] * K] * 4
    case, shared = prefix_case(6, [200] * 4, tails, 2, 2, 64, 16, dtype, sigma=1.0)
    q, k, v, table, lens = case
    k, v = k.clone(), v.clone()
    prefix = [table[i * K].long()[:13] for i in range(4)]
    q[:K] = q[:K].abs() + 0.1
    k[prefix[0], 0] = NONE                              # group 0, head 0: nothing of the prefix counts, and the rows' own tokens do not
    for b in range(K):
        k[table[b, 12].long(), 0] = NONE
    q[2 * K:3 * K] *= 100                               # group 2: scores of hundreds
    v[prefix[3][3], 1, 5, 7] = float("inf")             # group 3, head 1, one value: an infinity there for every row
    out, lse = prefixed((q, k, v, table, lens), shared)
    assert (out[:K, 0] == 0).all() and (lse[:K, 0] == NONE).all() and torch.isfinite(out[:K, 1]).all()
    assert (out[3 * K:, 1, 7] == float("inf")).all() and (~torch.isfinite(out)).sum() == K
    kk, vv = k.clone(), v.clone()
    kk[prefix[0], 0] = 0
    for b in range(K):
        kk[table[b, 12].long(), 0] = 0
    vv[prefix[3][3], 1, 5, 7] = 0
    ref, rlse = prefixed((q, kk, vv, table, lens), shared)
    other = torch.ones_like(out, dtype=torch.bool)
    other[:K, 0] = False
    other[3 * K:, 1, 7] = False
    assert torch.equal(out[other], ref[other]) and torch.equal(lse[K:], rlse[K:])
    check_attention("large", ref[2 * K:3 * K], rlse[2 * K:3 * K], q[2 * K:3 * K], kk, vv, table[2 * K:3 * K], lens[2 * K:3 * K])
    # NaN in one row's query, and in one row's own token
    q2, v2 = q.clone(), vv.clone()
    q2[K, 0, 3] = float("nan")
    v2[table[2 * K, 12].long(), 0, 10, 2] = float("nan")   # token 202 of the first row of group 2
    out2, _ = prefixed((q2, kk, v2, table, lens), shared)
    clean = torch.ones_like(out, dtype=torch.bool)
    clean[K, 0] = False
    clean[2 * K, 0, 2] = False
    assert torch.isnan(out2[K, 0]).all() and torch.isnan(out2[2 * K, 0, 2]) and torch.equal(out2[clean], ref[clean])


def test_prefix_attention_cache_above_32_bits():
    Hq, Hkv, D, page = 4, 2, 128, 64
    per = Hkv * page * D * 2
    pages = (1 << 33) // per + 70
    k, v = (torch.empty(pages, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    g = gen(1)
    ids = [0, (1 << 31) // per - 1, (1 << 31) // per, (1 << 32) // per - 1, (1 << 32) // per, (1 << 33) // per, pages - 1]
    for i in ids:
        k[i], v[i] = rnd(g, Hkv, page, D).bfloat16(), rnd(g, Hkv, page, D).bfloat16()
    q = rnd(g, 3, Hq, D, dtype=torch.bfloat16)
    table = i32([ids, ids, ids])
    lens, shared = i32([7 * page, 6 * page + 5, 5 * page]), i32([6 * page])
    case = (q, k, v, table, lens)
    check_attention("far pages", *prefixed(case, shared), *case)


# ---------------------------------------------------------------- all together

class Search:
    """A beam search over a paged cache: plan, store, attention, selection, fork, copies; two sets of tables that change places."""

    def __init__(self, B=3, K=4, Hq=8, Hkv=2, D=64, page=8, prompt=(5, 40, 16), steps=24, V=500, layers=2):
        self.B, self.K, self.Hkv, self.D, self.page, self.V = B, K, Hkv, D, page, V
        R, W = B * K, -(-(max(prompt) + steps + 4) // page)
        self.pages = F = B * (-(-max(prompt) // page)) + R * (-(-steps // page) + 2) + 7
        z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
        self.lens, self.table, self.count = [z(R), z(R)], [z(R, W) - 1, z(R, W) - 1], [z(1), z(1), z(1)]
        self.free = torch.arange(F, dtype=torch.int32, device="cuda")
        self.count[0].fill_(F)
        self.add, self.cu, self.status, self.fork_status = z(R), z(R + 1), z(1), z(1)
        self.positions, self.slots = z(R), torch.zeros(R, dtype=torch.int64, device="cuda")
        self.planned, self.copies, self.shared = z(R), z(3, R), z(B)
        self.cache = [torch.zeros(layers, F, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        self.qkv = torch.zeros(R, (Hq + 2 * Hkv) * D, device="cuda", dtype=torch.bfloat16)
        self.q, self.kx, self.vx = (x.unflatten(1, (-1, D)) for x in self.qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
        self.y, self.out = (torch.empty(R, Hq, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        self.freq = torch.from_numpy(10000.0 ** (-2.0 * np.arange(D // 2) / D)).cuda()
        self.logits, self.score = torch.zeros(R, V, device="cuda", dtype=torch.bfloat16), torch.zeros(B, K, device="cuda")
        self.score_new, self.token, self.parent = torch.zeros(B, K, device="cuda"), z(B, K), z(B, K)
        self.ws = [lb.alloc_beam_select_workspace(self.logits, self.score, K), lb.alloc_kv_fork_workspace(z(R), self.table[0], F),
                   lb.alloc_prefix_attn_workspace(self.q, self.cache[0][0], self.table[0], self.shared)]
        self.lse = torch.zeros(R, Hq, device="cuda")

    def start(self, prompt, g):
        """Prompts of one row a request, stored into both layers, and forked into beams."""
        B, K = self.B, self.K
        n = sum(prompt)
        i = lambda a: i32(a)
        lens, table = i([0] * B), self.table[1][:B]
        pos, slots = i([0] * n), torch.zeros(n, dtype=torch.int64, device="cuda")
        new, cu = i([0] * B), i([0] * (B + 1))
        lb.lory_kv_plan(lens, i(prompt), table, self.free, self.count[0], self.page, new, cu, pos, slots, self.count[1], self.status)
        x = rnd(g, n, self.Hkv, self.D, dtype=torch.bfloat16)
        q = rnd(g, n, self.q.shape[1], self.D, dtype=torch.bfloat16)
        for layer in range(self.cache[0].shape[0]):
            lb.lory_qk_rope_cache(q, x, x, pos, self.freq, self.cache[0][layer], self.cache[1][layer], slots)
        lb.lory_kv_fork(new, i(np.repeat(np.arange(B), K)), table, self.free, self.count[1], self.page, self.pages, self.lens[0],
                        self.table[0], self.count[0], self.copies, self.fork_status)
        lb.lory_kv_copy(*self.cache, self.copies)
        self.shared.copy_(i(prompt))
        self.score[:, 1:] = NONE

    def step(self, a, b):
        """From set a to set b."""
        self.attend(a)
        self.choose(a, b)

    def attend(self, a):
        lb.lory_kv_plan(self.lens[a], self.add, self.table[a], self.free, self.count[0], self.page, self.planned, self.cu, self.positions,
                        self.slots, self.count[1], self.status)
        for layer in range(self.cache[0].shape[0]):
            lb.lory_qk_rope_cache(self.q, self.kx, self.vx, self.positions, self.freq, self.cache[0][layer], self.cache[1][layer],
                                  self.slots, q_out=self.y)
        lb.lory_prefix_attn(self.y, self.cache[0][1], self.cache[1][1], self.table[a], self.planned, self.shared, out=self.out, lse=self.lse,
                            workspace=self.ws[2])

    def choose(self, a, b):
        self.logits += self.out.flatten(1).float().sum(1, keepdim=True).bfloat16()
        lb.lory_beam_select(self.logits, self.score, self.K, score_out=self.score_new, token=self.token, parent=self.parent,
                            workspace=self.ws[0])
        lb.lory_kv_fork(self.planned, self.parent.view(-1), self.table[a], self.free, self.count[1], self.page, self.pages, self.lens[b],
                        self.table[b], self.count[0], self.copies, self.fork_status, workspace=self.ws[1])
        lb.lory_kv_copy(*self.cache, self.copies)
        self.score.copy_(self.score_new)

    def rows(self, a):
        """Keys and values of every row of set a, in both layers."""
        out = []
        for b, n in enumerate(self.lens[a].tolist()):
            pages = self.table[a][b].long()[:-(-n // self.page)]
            out.append([x[:, pages].transpose(1, 2).flatten(2, 3)[:, :, :n] for x in self.cache] if n else [])
        return out


def feed(s, g):
    """What a model would compute: new queries, keys and values, and logits."""
    qkv, logits = rnd(g, *s.qkv.shape, dtype=torch.bfloat16), (3 * rnd(g, *s.logits.shape)).bfloat16()
    return qkv, logits


def test_beam_search_over_the_cache():
    """A search with ended beams against dense copies of every row's keys and values; pages are neither lost nor shared wrongly."""
    prompt, g = (5, 40, 16), gen(0)
    s = Search(prompt=prompt)
    s.start(prompt, g)
    R, K = s.B * s.K, s.K
    s.add.fill_(1)
    dense = s.rows(0)
    assert s.lens[0].tolist() == np.repeat(prompt, K).tolist() and s.fork_status.item() == 0
    for b in range(R):     # all beams of a request have its prompt
        assert all(torch.equal(x, y) for x, y in zip(dense[b], dense[b // K * K]))
    for step in range(24):
        a, b = step % 2, 1 - step % 2
        qkv, logits = feed(s, g)
        s.qkv.copy_(qkv)
        s.logits.copy_(logits)
        if step == 9:
            s.score[1, 1:] = NONE                      # all beams of request 1 but one have ended
        if step == 15:
            s.logits[:, 2:] = NONE                     # two tokens may follow: fewer candidates than beams for some
        score = s.score.clone()
        s.attend(a)
        if step % 8 == 0:   # before pages change hands
            check_attention(f"step {step}", s.out, s.lse, s.y, s.cache[0][1], s.cache[1][1], s.table[a], s.planned)
        s.choose(a, b)
        assert s.status.item() == 0 and s.fork_status.item() == 0
        check_select(f"step {step}", s.logits, score, K, (s.score_new, s.token, s.parent))
        k_new, v_new = lb.lory_qk_rope(s.q, s.kx, s.positions, s.freq)[1], s.vx
        grown = [[torch.cat([x, n[r][None, :, None].expand(2, -1, -1, -1)], 2) for x, n in zip(dense[r], (k_new, v_new))] if dense[r] else []
                 for r in range(R)]
        dense = [grown[p] if p >= 0 else [] for p in s.parent.view(-1).tolist()]
        for r, (x, y) in enumerate(zip(s.rows(b), dense)):
            assert len(x) == len(y) and all(torch.equal(m, n) for m, n in zip(x, y)), (step, r)
        # rows without a token add none, and theirs are not a plan's any more
        s.add.copy_((s.lens[b] > 0).int())
        if (s.lens[b] == 0).any():
            break
        used = {p for r, n in enumerate(s.lens[b].tolist()) for p in s.table[b][r, :-(-n // s.page)].tolist()}
        free = s.free[:s.count[0].item()].tolist()
        assert len(set(free)) == len(free) and not used & set(free) and len(used) + len(free) == s.pages
        last = [s.table[b][r, (n - 1) // s.page].item() for r, n in enumerate(s.lens[b].tolist()) if n % s.page]
        assert len(set(last)) == len(last)             # a page that is written next belongs to one row
    assert step >= 15


def test_search_on_another_stream_and_in_a_graph():
    """Two steps, there and back between the sets, run eagerly, on a side stream and from a graph; every replay against the eager run."""
    prompt, g = (5, 40, 16), gen(1)
    searches = [Search(prompt=prompt, steps=40) for _ in range(3)]
    for s in searches:
        s.start(prompt, gen(2))
        s.add.fill_(1)
    eager, side, captured = searches
    warm = Search(prompt=prompt)
    warm.start(prompt, gen(2))
    warm.step(0, 1)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    keep = [x.clone() for x in (captured.free, captured.score)]
    with torch.cuda.graph(graph):
        captured.step(0, 1)
        captured.step(1, 0)
    assert torch.equal(keep[0], captured.free) and torch.equal(keep[1], captured.score)
    for i in range(15):
        qkv, logits = feed(eager, g)
        for s in searches:
            s.qkv.copy_(qkv)
            s.logits.copy_(logits)
        eager.step(0, 1)
        eager.step(1, 0)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            side.step(0, 1)
            side.step(1, 0)
        torch.cuda.current_stream().wait_stream(stream)
        graph.replay()
        junk = torch.randn(1000, 1000, device="cuda")
        (junk @ junk).sum().item()
        for s in (side, captured):
            for n in ("free", "status", "fork_status", "positions", "slots", "planned", "copies", "y", "out", "lse", "logits", "score", "token",
                      "parent"):
                assert torch.equal(getattr(s, n), getattr(eager, n)), (i, n)
            for n in ("lens", "table", "count", "cache"):
                assert all(torch.equal(x, y) for x, y in zip(getattr(s, n), getattr(eager, n))), (i, n)
        assert eager.status.item() == 0 and eager.fork_status.item() == 0
    assert eager.lens[0].tolist() == (np.repeat(prompt, 4) + 30).tolist()


def test_event_timing_knows_the_operators_of_a_search():
    s = Search()
    s.start((5, 40, 16), gen(0))
    lb.lory_profile_read()
    lb.lory_profile_enable(True)
    try:
        s.step(0, 1)
        got = {r["name"]: r for r in lb.lory_profile_read()}
    finally:
        lb.lory_profile_enable(False)
    assert set(got) == {"qk_rope", "kv_plan", "beam_select", "kv_fork", "kv_copy", "prefix_attn"}
    assert all(got[n]["launches"] == 1 and got[n]["ms"] > 0 for n in ("beam_select", "kv_fork", "kv_copy", "prefix_attn"))
    assert got["beam_select"]["bytes"] == 12 * 500 * 2


@pytest.mark.parametrize("dtype", [torch.float32])
def test_beam_example(dtype):
    """The example's search: its beams' scores are those of their tokens, run one by one as rows of their own."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate_beams.py")
    spec = importlib.util.spec_from_file_location("generate_beams", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    block = m.Block(d=64, heads=4, kv_heads=2, head_dim=16, d_ff=128, experts=4, dtype=dtype)
    g = gen(4)
    B, L, K, V, steps, page = 3, 21, 4, 90, 9, 8
    head = (rnd(g, block.d, V) * block.d ** -0.5).to(dtype)
    prompts, lens = rnd(g, B, L, block.d).to(dtype), i32([5, 21, 16])
    score, tokens, status, count = m.search(block, prompts, lens, head, K, steps, page)
    assert [s.item() for s in status] == [0, 0] and tokens.shape == (B, K, steps) and (tokens >= 0).all()
    assert len({tuple(t) for t in tokens[1].tolist()}) == K and (score[:, 1:] <= score[:, :-1]).all()
    # pages in use: of the prompts' whole pages one set a request, and at most ceil(steps / page) + 1 a beam
    pages = B * -(-L // page) + B * K * (-(-steps // page) + 2)
    assert count.item() >= pages - sum(-(-n // page) for n in lens.tolist()) - B * K * (-(-steps // page) + 1)
    for k in range(K):      # beam k of every request as a batch of single rows
        r = m.Requests(block, B, 60, page, L + steps)
        h, merged = m.prefill(block, r, prompts, lens)
        h = m.next_input(h[torch.arange(B, device="cuda"), lens.long() - 1])
        total = torch.zeros(B, dtype=torch.float64, device="cuda")
        one = m.Beams(r, lens, B, 1, 60)
        one.shared.zero_()
        for t in range(steps):
            token = tokens[:, k, t].long()
            total += torch.log_softmax((h @ head).double(), 1).gather(1, token[:, None])[:, 0]
            if t + 1 < steps:
                h = m.next_input(m.decode(block, one, m.next_input(head.T[token].contiguous()), merged))
        # fp32 all along; the merged FFN adds in another order for several tokens of a sequence.  A step's logits are sums of
        # 64 products of normalised states, off by at most a few hundred roundings of fp32 after the block: 9 steps of 1e-4
        assert (score[:, k].double() - total).abs().max().item() < 9e-4, k
