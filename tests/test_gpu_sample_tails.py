"""axon_sample where most of the vocabulary lies 26 to 31 nats below the largest logit: there the resolution of the weights
decides, 2^-44 of the largest.

With U units in the largest weight (it lies 0.5 to 1.5 steps of 2^(1/512) below 2^44: U >= 2^44 / 1.00204) a weight w of the formula
is held as an integer that is off by half a unit, by 0.5004 where it becomes 0, and by 2^-41 of w: by W = 1.003 * 2^-45 + 2^-41 w of
the largest. A sum of n of them is off by E = n 1.003 * 2^-45 + 2^-41 of itself. The share asked for of a sum,
or the draw's, adds a unit for its rounding and as much error as the sum: 2 E + 2^-43 in all on either side of a border.
Hence the tokens that stay after top-p are the first n of the order with n between those that the share needs with that much
less and more, a weight stays by min-p if it is above min_p + W and goes if it is below min_p - W, and the token drawn is one
whose stretch of the running sum the draw comes that near to. The probability is w / S of an S among these, off by
W / S and by fp32's 2^-24."""
import numpy as np
import pytest

from test_gpu_sample import DEV, ax  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
HALF = 1.003 * 2.0 ** -45


def allowed(row, temp, p, m, u, token, prob):
    """Asserts that a row's answer is within the bounds above."""
    row = np.asarray(row, dtype=np.float64)
    w = np.exp((row - row.max()) / np.float64(temp))
    V = len(w)
    order = np.lexsort((np.arange(V), -row))
    c = np.cumsum(w[order])
    off = 2 * (V * HALF + 2.0 ** -41 * c[-1]) + 2.0 ** -43
    few = many = V  # of the order, certainly and possibly
    if p < 1:
        few, many = (min(V, 1 + int(np.searchsorted(c, p * c[-1] + x))) for x in (-off, off))
    sure, maybe = (np.zeros(V, dtype=bool) for _ in range(2))
    sure[order[:few]] = True
    maybe[order[:many]] = True
    if m > 0:
        slack = HALF + 2.0 ** -41 * m
        sure &= w >= m + slack
        maybe &= w >= m - slack
    sure[order[0]] = maybe[order[0]] = True
    assert maybe[token]
    low, high = np.cumsum(np.where(sure, w, 0.0)), np.cumsum(np.where(maybe, w, 0.0))
    assert u * low[-1] <= high[token] + off, "drawn too early"
    assert (low[token - 1] if token else 0.0) <= u * high[-1] + off, "drawn too late"
    one = HALF + 2.0 ** -41 * w[token]
    assert (w[token] - one) / (high[-1] + off) * (1 - 2.0 ** -24) <= prob <= (w[token] + one) / (low[-1] - off) * (1 + 2.0 ** -24)
    return int(sure.sum()), int(maybe.sum())


def tail(V, top, low, high, seed):
    r = np.random.default_rng(seed)
    row = r.uniform(low, high, V).astype(np.float32)
    row[top] = 0.0
    return row


ROWS = [(524287, -31, -31, 0.0), (524287, -31, -31, 2.4e-8), (524287, -31, -31, 1.1e-8), (0, -31, -31, 0.99999994), (0, -31, -31, 0.5),
        (524287, -31, -30, 3e-8), (70000, -31, -30, 1e-8), (70000, -31, -30, 0.99999994), (300000, -30.9, -29, 6e-8),
        (5, -35, -26, 4e-7), (5, -35, -26, 0.9999995)]
CUTS = [(1.0, 0.0), (1 - 2.0 ** -24, 0.0), (1 - 2.0 ** -23, 0.0), (0.99999, 0.0), (1.0, 1e-12), (1.0, 5e-14), (1 - 2.0 ** -23, 1e-13)]


@pytest.mark.parametrize("p,m", CUTS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,temp", [(524288, 1.0), (128257, 1.0), (128257, 0.93)])
def test_many_small_weights(ax, V, temp, dtype, p, m):  # noqa: F811
    rows = [tail(V, min(top, V - 1), low, high, i) for i, (top, low, high, _) in enumerate(ROWS)]
    x = torch.from_numpy(np.stack(rows)).to(DEV, torch.float32 if dtype == "fp32" else torch.bfloat16)
    u = torch.tensor([r[3] for r in ROWS], dtype=torch.float32, device=DEV)
    B = len(rows)
    full = lambda v: torch.full((B,), v, dtype=torch.float32, device=DEV)  # noqa: E731
    tokens, prob = torch.full((B,), -7, dtype=torch.int32, device=DEV), full(float("nan"))
    ax.axon_sample(x, u, tokens, temperature=full(temp), top_p=full(p), min_p=full(m), prob=prob)
    x, t, q = x.float().cpu().numpy(), full(temp)[0].item(), (full(p)[0].item(), full(m)[0].item())
    for b in range(B):
        allowed(x[b], t, *q, u[b].item(), int(tokens[b]), float(prob[b]))


def test_what_is_below_half_a_unit_is_never_drawn(ax):  # noqa: F811
    """Weights of 2^-46 and less are 0: with the largest logit last, and nothing else of a weight, every draw takes it."""
    V, B = 100000, 8
    x = torch.full((B, V), -46 * 0.6931472, device=DEV)
    x[:, -1] = 0.0
    u = torch.tensor([0.0, 1e-30, 1e-12, 1e-9, 1e-7, 0.1, 0.9, 1.0], device=DEV)
    tokens, prob = torch.empty(B, dtype=torch.int32, device=DEV), torch.empty(B, device=DEV)
    ax.axon_sample(x, u, tokens, prob=prob)
    assert (tokens == V - 1).all() and (prob == 1).all()
