"""Tokens from logits (axon_sample) against sorting and running sums in 64 bits on the host.

The token has to be the same: both sides decide by sums that are exact to 2^-40 of the total, and the tests' random
numbers and shares stay 1e-9 clear of every border that they are compared with (checked on the reference's side; numbers at
a border on purpose have exact sums on both). The probability is a quotient of two such sums, rounded to fp32: 2^-24 of
it, and 2^-40 of the total from its weight, 2^-23 allowed in all."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ax():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


def clear_of(borders, at, total):
    return np.abs(np.asarray(borders) - at).min() > 1e-9 * total


def reference(row, temp, k, p, m, u):
    """(token, probability, whether every decision is clear of its border)."""
    row = np.where(np.isnan(row), -np.inf, np.asarray(row, dtype=np.float64))
    best = int(row.argmax())
    if row[best] == -np.inf:
        return -1, 0.0, True
    if not temp > 0:
        return best, 1.0, True
    if row[best] == np.inf:
        row = np.where(row == np.inf, 0.0, -np.inf)
    with np.errstate(over="ignore"):
        w = np.exp((row - row[best]) / np.float64(temp))
    order = np.lexsort((np.arange(len(row)), -row))
    sure = True
    if 0 < k < len(row):
        order = order[:k]
    if p < 1:
        c = np.cumsum(w[order])
        at = max(np.float64(p), 0.0) * c[-1]
        sure &= clear_of(c, at, c[-1])
        order = order[:1 + int(np.searchsorted(c, at))]
    if m > 0:
        sure &= np.abs(w[order] - m).min() > 1e-9 * m
        order = order[(w[order] >= m) | (np.arange(len(order)) == 0)]
    order = np.sort(order)
    c = np.cumsum(w[order])
    u = min(max(np.float64(u), 0.0), 1 - 2.0 ** -24)
    if u > 0:
        sure &= clear_of(c, u * c[-1], c[-1])
    i = int(np.searchsorted(c, u * c[-1], side="right"))
    return int(order[i]), w[order[i]] / c[-1], sure


def f32(v, B):
    return torch.tensor(np.broadcast_to(np.asarray(v, dtype=np.float32), (B,)).copy(), device=DEV)


def sample(ax, x, u, temp=None, k=None, p=None, m=None, **kw):
    B = x.shape[0]
    tok = torch.full((B,), -7, dtype=torch.int32, device=DEV)
    prob = torch.full((B,), float("nan"), device=DEV)
    ax.axon_sample(x, f32(u, B), tok, temperature=None if temp is None else f32(temp, B),
                   top_k=None if k is None else torch.tensor(np.broadcast_to(k, (B,)).copy(), dtype=torch.int32, device=DEV),
                   top_p=None if p is None else f32(p, B), min_p=None if m is None else f32(m, B), prob=prob, **kw)
    return tok.cpu().numpy(), prob.double().cpu().numpy()


def check(ax, x, u, temp=None, k=None, p=None, m=None, least=0.9):
    """least: part of the rows whose decisions have to be clear of every border, by the choice of inputs."""
    B = x.shape[0]
    tok, prob = sample(ax, x, u, temp, k, p, m)
    rows = x.double().cpu().numpy()
    row = lambda v, d, b: d if v is None else np.broadcast_to(np.asarray(v), (B,))[b]  # noqa: E731
    asked = 0
    for b in range(B):
        single = lambda v, d: float(np.float32(row(v, d, b)))  # noqa: E731
        want, wp, sure = reference(rows[b], single(temp, 1.0), int(row(k, 0, b)), single(p, 1.0), single(m, 0.0), single(u, 0.0))
        if sure:
            asked += 1
            assert tok[b] == want, (b, tok[b], want)
            assert abs(prob[b] - wp) <= 2.0 ** -23 * wp, (b, prob[b], wp)
    assert asked >= least * B, f"{asked} of {B} rows are clear of their borders"


def logits(B, V, seed, std=2.0, likely=20, dtype=torch.float32):
    r = np.random.default_rng(seed)
    x = r.standard_normal((B, V)) * std
    for b in range(B):
        at = r.integers(0, V, min(likely, V))
        x[b, at] += 6 + 6 * r.random(len(at))
    return torch.from_numpy(x.astype(np.float32)).to(DEV).to(dtype), r.random(B).astype(np.float32)


SIZES = [1, 2, 5, 31, 33, 257, 1000, 2047, 32000, 50257, 151936]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("B", [1, 5])
def test_temperature_alone(ax, V, B):
    x, u = logits(B, V, seed=V + B)
    check(ax, x, u, temp=[0.5, 0.8, 1.0, 1.5, 30.0][:B])


@pytest.mark.parametrize("V", SIZES)
def test_top_k(ax, V):
    ks = [1, 2, 3, 7, 50, 200, 1023, 1024, 1025, 4000, V - 1, V, V + 1, 0, -3]
    x, u = logits(len(ks), V, seed=V)
    check(ax, x, u, temp=1.3, k=ks)


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("std", [1.3, 4.0])
def test_top_p(ax, V, std):
    ps = [1e-6, 0.01, 0.1, 0.3, 0.5, 0.9, 0.95, 0.999, 0.99999, 1.0, 1.5]
    x, u = logits(len(ps), V, seed=V + 1, std=std, likely=0)
    check(ax, x, u, temp=1.0, p=ps)


@pytest.mark.parametrize("V", SIZES)
def test_min_p(ax, V):
    ms = [1e-9, 1e-4, 0.01, 0.05, 0.3, 0.999, 1.7, 0.0, -1.0]
    x, u = logits(len(ms), V, seed=V + 2)
    check(ax, x, u, temp=0.9, m=ms)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [777, 32000, 49152])
def test_all_together(ax, V, dtype):
    B = 48
    x, u = logits(B, V, seed=V + 3, dtype=dtype)
    r = np.random.default_rng(V)
    check(ax, x, u, temp=r.uniform(0.2, 2.0, B), k=r.integers(0, 400, B), p=r.uniform(0.2, 1.1, B),
          m=np.where(r.random(B) < 0.5, r.uniform(0.0, 0.1, B), 0.0))


@pytest.mark.parametrize("B", [17, 33, 70, 160, 400])
def test_batches(ax, B):
    x, u = logits(B, 8000, seed=B)
    check(ax, x, u, temp=0.8, k=40, p=0.9)
    check(ax, x, u, temp=1.1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_many_equal_logits(ax, dtype):
    """Few values: cuts fall into thousands of equal logits, of which the lowest numbers stay. Every weight is a power
    of two, so both sides' sums are exact."""
    r = np.random.default_rng(11)
    V, B = 30000, 24
    x = torch.from_numpy(-r.integers(0, 4, (B, V)).astype(np.float32)).to(DEV).to(dtype)
    rows = x.double().cpu().numpy()
    temp = float(np.float32(1 / np.log(2)))  # weights 2^-d but for a rounding of the temperature
    ks = r.integers(1, V, B)
    u = r.random(B).astype(np.float32)
    tok, _ = sample(ax, x, u, temp=temp, k=ks)
    tok_p, _ = sample(ax, x, u, temp=temp, p=(ks / V).astype(np.float32))
    for b in range(B):
        for got, kk, pp in ((tok[b], int(ks[b]), 1.0), (tok_p[b], 0, float(np.float32(ks[b] / V)))):
            want, _, sure = reference(rows[b], temp, kk, pp, 0.0, float(u[b]))
            if sure:
                assert got == want


@pytest.mark.parametrize("crowd", [200, 900, 3000, 20000])
@pytest.mark.parametrize("B,V", [(2, 50257), (40, 33000)])
@pytest.mark.parametrize("values", [0, 5])
def test_a_crowd_within_a_thirtieth_of_an_octave(ax, B, V, crowd, values):
    """Cuts and draws among many logits whose weights differ by 1.5 % at most; values: of so many different logits."""
    r = np.random.default_rng(crowd + V + values)
    x = (r.standard_normal((B, V)) - 9).astype(np.float32)
    for b in range(B):
        at = r.permutation(V)[:crowd]
        x[b, at] = 4 + 0.015 * (r.integers(0, values, crowd) / values if values else r.random(crowd))
    x, u = torch.from_numpy(x).to(DEV), r.random(B).astype(np.float32)
    part = r.uniform(0.1, 0.9, B)
    check(ax, x, u, p=part)
    check(ax, x, u, k=np.maximum(1, (part * crowd).astype(np.int32)))
    check(ax, x, u, k=np.maximum(1, (part * crowd).astype(np.int32)), p=r.uniform(0.2, 0.9, B))
    check(ax, x, u, p=part, m=0.9949 if values == 0 else 0.9925)


def test_borders_go_to_the_next_token(ax):
    x = torch.zeros(1, 8, device=DEV)
    for u, want in [(0.0, 0), (0.125, 1), (0.12499999, 0), (0.5, 4), (0.99999994, 7), (1.0, 7), (2.0, 7), (-1.0, 0), (float("nan"), 0)]:
        assert sample(ax, x, u)[0][0] == want, u
    for p, n in [(0.125, 1), (0.1250001, 2), (0.5, 4), (0.9, 8), (0.0, 1), (-1.0, 1), (1e-30, 1)]:
        assert sample(ax, x, 0.99999994, p=p)[0][0] == n - 1, p
        assert sample(ax, x, 0.0, p=p)[1][0] == np.float32(1 / n)
    for k in range(1, 9):
        assert sample(ax, x, 0.99999994, k=k)[0][0] == k - 1


def test_equal_logits_of_the_whole_vocabulary(ax):
    V = 151936
    x = torch.full((3, V), -2.5, device=DEV)
    u = np.array([0.0, 0.5, 0.75], dtype=np.float32)
    for k in (1, 1000, 100000):
        assert sample(ax, x, u, k=k)[0].tolist() == [0, k // 2, 3 * k // 4]
    assert sample(ax, x, u, p=0.5)[0].tolist() == [0, V // 4, 3 * V // 8]
    assert sample(ax, x, u, k=100000, p=0.25)[0].tolist() == [0, 12500, 18750]


def test_greedy_rows(ax):
    x, u = logits(6, 50257, seed=4)
    x[1, 700] = x[1, 40000] = 50.0
    x[2, 50256] = 50.0
    tok, prob = sample(ax, x, u, temp=[0.0, 0.0, -1.0, float("nan"), 0.0, 0.0], k=3, p=0.1, m=0.5)
    want = x.double().cpu().numpy().argmax(1)
    assert want[1] == 700 and tok.tolist() == want.tolist() and (prob == 1).all()


def test_masked_rows(ax):
    inf, nan = float("inf"), float("nan")
    x, u = logits(8, 1000, seed=5)
    x[0] = -inf
    x[1] = nan
    x[2] = -inf
    x[2, 999] = -1e30
    x[3, ::2] = -inf
    x[4, 1:] = nan
    x[5, [3, 800]] = inf
    x[6] = torch.finfo(torch.float32).min
    x[7, 5:] = torch.finfo(torch.float32).min
    u[5] = 0.75
    for kw in (dict(), dict(k=5), dict(p=0.8), dict(m=0.2), dict(temp=0.0)):
        tok, prob = sample(ax, x, u, **kw)
        assert tok[:3].tolist() == [-1, -1, 999] and prob[:3].tolist() == [0, 0, 1]
        assert tok[4] == 0 and tok[5] == (3 if "temp" in kw or "p" in kw and kw["p"] < 0.5 else 800)
        assert tok[7] < 5
    check(ax, x[3:4], u[3:4], temp=1.0, least=1)
    check(ax, x[6:7], u[6:7], temp=1.0, p=0.37, least=1)


def test_extreme_temperatures(ax):
    x, u = logits(5, 5000, seed=6)
    check(ax, x, u, temp=[1e-30, 1e-3, 1e4, 1e30, float("inf")])
    check(ax, x, u, temp=[1e-30, 1e-3, 1e4, 1e30, 3e38], k=1234, p=0.4)


def test_strides_and_odd_rows(ax):
    V, B = 5003, 6
    x, u = logits(B, V, seed=7)
    for dtype in (torch.float32, torch.bfloat16):
        for wide, off in ((V, 0), (V + 1, 1), (V + 13, 3), (V + 16, 8)):
            big = torch.full((B, wide), 1e4, device=DEV).to(dtype)  # read behind a row and it wins
            big[:, off:off + V] = x.to(dtype)
            check(ax, big[:, off:off + V], u, temp=0.9, k=300, p=0.95)


def test_largest_vocabulary(ax):
    V = 524288
    x, u = logits(2, V, seed=8)
    x[0, V - 1] = 40.0
    check(ax, x, u, temp=1.0, p=0.9, least=0.5)
    check(ax, x, u, temp=2.0, k=1000, least=0.5)


def test_counts_follow_the_weights(ax):
    """20,000 draws from one row: each token's count within 6 standard deviations."""
    n = 20000
    x = torch.tensor([[1.0, 0.0, 3.0, 2.0, -1.0, 2.5]], device=DEV).repeat(n, 1)
    u = torch.rand(n, generator=torch.Generator().manual_seed(1)).numpy()
    tok, _ = sample(ax, x, u, k=4)
    w = np.exp([1.0, 0, 3.0, 2.0, 0, 2.5]) * np.array([1, 0, 1, 1, 0, 1])
    w /= w.sum()
    got = np.bincount(tok, minlength=6)
    assert (np.abs(got - n * w) <= 6 * np.sqrt(n * w * (1 - w))).all()


def test_same_answer_every_time_and_captured(ax):
    x, u = logits(40, 30000, seed=9)
    args = dict(temperature=f32(0.9, 40), top_p=f32(0.97, 40), top_k=torch.full((40,), 5000, dtype=torch.int32, device=DEV))
    ud, tok, prob = f32(u, 40), torch.empty(40, dtype=torch.int32, device=DEV), torch.empty(40, device=DEV)
    ax.axon_sample(x, ud, tok, prob=prob, **args)
    first, pf = tok.clone(), prob.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ax.axon_sample(x, ud, tok, prob=prob, **args)
    for _ in range(5):
        tok.zero_()
        g.replay()
        assert torch.equal(tok, first) and torch.equal(prob, pf)
    ud.fill_(0.0)
    g.replay()
    assert not torch.equal(tok, first)


def test_two_calls_at_once(ax):
    """Calls on two streams share nothing."""
    x, u = logits(20, 60000, seed=10)
    y, v = logits(20, 60000, seed=12)
    want = sample(ax, x, u, temp=1.0, p=0.9)[0], sample(ax, y, v, temp=1.0, p=0.9)[0]
    ud, vd, t, p = f32(u, 20), f32(v, 20), f32(1.0, 20), f32(0.9, 20)
    a, b = (torch.empty(20, dtype=torch.int32, device=DEV) for _ in range(2))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(s1):
            ax.axon_sample(x, ud, a, temperature=t, top_p=p)
        with torch.cuda.stream(s2):
            ax.axon_sample(y, vd, b, temperature=t, top_p=p)
    torch.cuda.synchronize()
    assert a.cpu().numpy().tolist() == want[0].tolist() and b.cpu().numpy().tolist() == want[1].tolist()
