"""Selection over rows that a workgroup streams in several whole steps: barred tokens, jumps and orders that its reference of the
exponentials, its bound and its lists of candidates have to follow.

Bounds are those of check_select in test_beam_gpu.py.  They hold here too: an exponential's argument is taken from a reference that is at most
24 below the logits that count (64 at most by the kernel's rule), so its rounding is 22 x 2^-24 at most beside the 34 of a group's sum and the exponential."""
import pytest
import torch

from paper_2405_03133_amd import binding as lb
from test_attn_gpu import T, gen
from test_beam_gpu import NONE, check_select, logits_of, select

pytestmark = pytest.mark.gpu

PER = {"bf16": 8, "f32": 4}                       # logits of a 16-byte vector
CHUNKS = 16                                       # of a row where rows are few
VECTORS = 4096                                    # of a chunk in these tests: four whole steps of 1024, and nothing behind them
LOW = {"far": -1e4, "billion": -1e9, "lowest": None, "none": NONE}


def low(name, dtype):
    return torch.finfo(T[dtype]).min if LOW[name] is None else LOW[name]


def long_rows(g, rows, dtype, sigma=2.0):
    return logits_of(g, rows, CHUNKS * VECTORS * PER[dtype], dtype, sigma)


def by_vector(x, dtype):
    """[rows, chunks, vectors of a chunk, logits of a vector], the same memory."""
    return x.view(x.shape[0], CHUNKS, VECTORS, PER[dtype])


def of_wavefront(w):
    """Vectors of a chunk that wavefront w of a workgroup reads."""
    return (torch.arange(VECTORS, device="cuda") % 256) // 64 == w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("barred", list(LOW))
@pytest.mark.parametrize("shift", [0.0, -200.0, 100.0])
def test_select_where_a_wavefront_starts_barred(barred, shift, dtype):
    """The first step of one wavefront, of two, and of all but one has only barred tokens; what comes later is ordinary, and most
    of it no candidate."""
    g = gen(7)
    R, K, k = 3, 4, 6
    x = by_vector(long_rows(g, R * K, dtype), dtype)
    x += shift
    first = torch.arange(VECTORS, device="cuda") < 1024
    for r in range(R * K):
        waves = [[r % 4], [r % 4, (r + 1) % 4], [w for w in range(4) if w != r % 4]][r // 4]
        for w in waves:
            x[r, :, first & of_wavefront(w)] = low(barred, dtype)
    # and the best tokens all in the first step of the others: a bound that the wavefront's own logits stay below
    x[:, :, 1024:] = torch.minimum(x[:, :, 1024:], torch.tensor(shift + 4.0, device="cuda", dtype=T[dtype]))
    check_select(f"{barred} {shift}", x.view(R * K, -1), -torch.rand(R, K, generator=g, device="cuda"), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("barred", list(LOW))
@pytest.mark.parametrize("R,K,V,k", [(130, 4, 32000, 4), (18, 8, 128000, 8)])
def test_select_where_few_tokens_are_allowed(R, K, V, k, barred, dtype):
    """A constraint: twenty tokens anywhere, or two runs of them, of every row."""
    g = gen(V + k)
    full = logits_of(g, R * K, V, dtype)
    allowed = torch.zeros(R * K, V, dtype=torch.bool, device="cuda")
    allowed.scatter_(1, torch.randint(0, V, (R * K, 20), generator=g, device="cuda"), True)
    allowed[::3, 30200:31200] = True
    allowed[::3, :1000] = True
    x = torch.where(allowed, full, torch.tensor(low(barred, dtype), device="cuda", dtype=T[dtype]))
    check_select(f"few allowed, {barred}", x, -torch.rand(R, K, generator=g, device="cuda"), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_after_a_low_prefix(dtype):
    """Logits that jump by more than fp32's exponentials hold, once and again, at places that differ from row to row."""
    g = gen(11)
    R, K = 2, 4
    x = long_rows(g, R * K, dtype)
    n = x.shape[1]
    at = torch.arange(n, device="cuda") % (n // CHUNKS)
    for r in range(R * K):
        x[r] -= 150.0 * ((at < 9000 + 1000 * r).float() + (at < 5000 + 500 * r).float()).to(T[dtype])
    check_select("two jumps", x, torch.zeros(R, K, device="cuda"), 8)
    check_select("two falls", x.flip(1).contiguous(), torch.zeros(R, K, device="cuda"), 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_nan_among_barred_tokens(dtype):
    """A wavefront meets a NaN before its first number: the beam has no candidates, and the others keep theirs."""
    g = gen(13)
    R, K = 3, 4
    x = by_vector(long_rows(g, R * K, dtype), dtype)
    at = torch.arange(VECTORS, device="cuda")
    odd = []
    for r in range(R * K):
        w = r % 4
        x[r, 5, (at < 2048) & of_wavefront(w)] = NONE
        if r % K != r // K:
            continue
        x[r, 5, 1024 + 64 * w + 11, PER[dtype] - 1] = float("nan")
        odd.append(r)
    x = x.view(R * K, -1)
    score = -torch.rand(R, K, generator=g, device="cuda")
    check_select("NaN among -inf", x, score, 8)
    _, _, parent = select(x, score, 8)
    assert not torch.isin(parent, torch.tensor(odd, device="cuda", dtype=torch.int32)).any()


def steps_per_vocab(dtype, order, V, k):
    """Seconds of a call on a row whose logits come in that order, the best of a few."""
    x = torch.linspace(-10.0, 10.0, V, device="cuda", dtype=torch.float64).to(T[dtype])[None]
    x = {"up": x, "down": x.flip(1)}[order].contiguous()
    score, best = torch.zeros(1, 1, device="cuda"), []
    ws = lb.alloc_beam_select_workspace(x, score, k)
    for _ in range(4):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        lb.lory_beam_select(x, score, k, workspace=ws)
        b.record()
        torch.cuda.synchronize()
        best.append(a.elapsed_time(b))
    check_select(f"{order} {V}", x, score, k)
    return min(best)


@pytest.mark.parametrize("order", ["up", "down"])
@pytest.mark.parametrize("dtype,k", [("bf16", 4), ("f32", 1), ("f32", 64)])
def test_select_of_sorted_logits(order, dtype, k):
    """Every vector beats all before it, and so does every one of a chunk: the time grows as the row does, not as its square
    (eight times the row: 64)."""
    V = 1 << 18 if dtype == "f32" else 1 << 19
    short, long = steps_per_vocab(dtype, order, V, k), steps_per_vocab(dtype, order, 8 * V, k)
    print(f"[beam] {order} {dtype} k {k}: {short * 1e3:.0f} us, {long * 1e3:.0f} us", flush=True)
    assert long <= 16 * short


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [1, 7, 64])
def test_select_of_equal_logits_in_long_rows(k, dtype):
    """Every vector of every step equals the bound: the lowest tokens of the first beam; and two values, the larger one rare."""
    R, K = 2, 2
    x = torch.zeros(R * K, CHUNKS * VECTORS * PER[dtype], device="cuda", dtype=T[dtype])
    score = torch.zeros(R, K, device="cuda")
    _, token, parent = select(x, score, k)
    assert (token == torch.arange(k, device="cuda")).all() and (parent == torch.tensor([[0], [K]], device="cuda")).all()
    g = gen(k)
    x[torch.rand(x.shape, generator=g, device="cuda") < 1e-5] = 0.5
    check_select("rare", x, score, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [8, 16, 64])
def test_select_of_more_equal_candidates_than_a_list_holds(K, dtype):
    """k equal candidates of every chunk of every beam, 8192 and more of a request: the first beam's, whatever list they came in;
    with different scores the best beam's."""
    k, V = 64, 40000
    x = torch.zeros(2 * K, V, device="cuda", dtype=T[dtype])
    score = torch.zeros(2, K, device="cuda")
    score[1, K - 2:] = 1.0
    _, token, parent = select(x, score, k)
    assert (token == torch.arange(k, device="cuda")).all() and (parent[0] == 0).all() and (parent[1] == 2 * K - 2).all()
    # ten better tokens of every beam, at other places in each: the sums are those of the same terms, rounded in another order, so
    # which beam comes first is the sums' affair
    n = torch.arange(10, device="cuda")
    for b in range(2 * K):
        x[b, (n * 3989 + 17 * b) % V] = 1.0
    check_select("few better ones", x, score, k)
