"""An infinite value at a visible token leaves its dim of the output not finite, with every attention on a paged cache and
in both types (fp16 saturates finite outputs only); the other dims are right, by the tolerances of the operators' own tests."""
import numpy as np
import pytest

import test_gpu_kv_attention as kv
import test_gpu_shared as sh
from test_gpu_kv_attention import ULP, ax  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
VALUES = [float("inf"), float("-inf")]
DIM = 5


def check(out, want, vmax, dtype, first, prob=0.0):
    """The first `first` heads of every row see the value."""
    out, rest = out.double().cpu().numpy(), [x for x in range(out.shape[2]) if x != DIM]
    assert not np.isfinite(out[:, :first, DIM]).any()
    got = np.concatenate([out[:, :, rest].ravel(), out[:, first:, DIM].ravel()])
    exp = np.concatenate([want[:, :, rest].ravel(), want[:, first:, DIM].ravel()])
    assert np.isfinite(got).all()
    assert (np.abs(got - exp) <= ULP[dtype] * np.abs(exp) + (5e-4 + prob) * vmax).all()


def spoil(c, value):
    """Token 3 of the first row's second block, kv head 0; the reference has 0 there, which its other dims do not see."""
    c.v[c.layer, int(c.table[0, 1]), 0, 3, DIM] = value


@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,d,past", [(4, 1, 64, 40), (8, 2, 128, 40), (16, 1, 64, 200), (8, 2, 128, 20000)])
def test_one_token(ax, H, G, d, past, dtype, value):  # noqa: F811
    c = kv.Case(H, G, d, dtype, [past], [1], 0, 0, seed=past)
    spoil(c, value)
    want, _ = c.reference()
    check(kv.run_decode(ax, c)[0], want, c.vmax(), dtype, H // G)


@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,d,past,new", [(8, 2, 128, 40, 7), (14, 2, 64, 300, 200), (8, 2, 128, 20000, 3)])  # the last: split
def test_chunks(ax, H, G, d, past, new, dtype, value):  # noqa: F811
    c = kv.Case(H, G, d, dtype, [past], [new], 0, 0, seed=past + new)
    spoil(c, value)
    out = torch.empty_like(c.q)
    ax.axon_attn_prefill(ax.make_kv_cache(c.k, c.v), c.layer, c.q, c.cu, c.ctx, new, out, block_table=c.bt, err=c.err)
    want, _ = c.reference()
    check(out, want, c.vmax(), dtype, H // G, kv.PROB[dtype])
    assert ax.axon_check_error(c.err) == (0, 0)


@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [3, 40])
def test_shared_prefixes(ax, rows, dtype, value, monkeypatch):  # noqa: F811
    monkeypatch.setenv("AXON_SHARED_MIN_BYTES", "0")
    c = sh.Case(8, 2, 128, dtype, [(1024, [1030 + 3 * i for i in range(rows)])], seed=rows)
    spoil(c, value)
    out, _ = sh.run(ax, c)
    want, _ = c.reference(range(rows))
    check(out, want, max(np.abs(v).max() for v in c.values), dtype, 4)
