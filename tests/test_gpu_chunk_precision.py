"""Rounding of the chunk attention: its probabilities enter the product with V in two 16-bit terms, so that
the output's own rounding is the only one that counts, as in the one-token attention; and a model
whose window keeps its first tokens visible, whose prompts take it, is no less exact than without them."""
import numpy as np
import pytest

from helpers import create
from test_gpu_attn_precision import N, S, SHAPE, V, _exact, _model
from test_gpu_kv_attention import TYPES, Case
from test_gpu_parity import _ax, run_prefill

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,d,past,new,window,sinks", [
    (9, 3, 64, [0], [16], 0, 0),                    # a short prompt: few keys, all in a masked step
    (8, 2, 128, [0], [300], 0, 0),                  # more keys than four steps for the last rows
    (8, 2, 64, [900, 40], [70, 200], 0, 0),         # chunks after a past
    (8, 2, 128, [300, 0, 700], [33, 260, 1], 200, 4),
    (8, 2, 128, [2500], [12], 0, 0),                # keys of an item shared by a cluster
])
def test_error_is_that_of_the_outputs_rounding(H, G, d, past, new, window, sinks, dtype):
    """rms error against 64 bits over the rms error of the exact result rounded once. Two terms leave 2^-17 (bf16) of a
    probability, nothing beside the output's 2^-9; scores are sums of at most 128 products whose partial sums stay
    below 64, cut at 2^-24 of them in each of eight steps: 3e-5 in the exponent at most, against 1.4e-4 rms of a
    rounding to fp16 (the quotient and the exponential add a few 2^-23): sqrt(1 + 0.05) at the very most, 1.03 allowed."""
    ax = _ax()
    c = Case(H, G, d, dtype, past, new, window, sinks, seed=41)
    out = torch.full_like(c.q, float("nan"))
    ax.axon_attn_prefill(ax.make_kv_cache(c.k, c.v), c.layer, c.q, c.cu, c.ctx, max(new), out, block_table=c.bt, window=window,
                         sinks=sinks, err=c.err)
    assert ax.axon_check_error(c.err) == (0, 0)
    want, _ = c.reference()
    once = torch.from_numpy(want).to(TYPES[dtype]).double().numpy()
    got = out.double().cpu().numpy()
    rms = [float(np.sqrt(np.mean((x - want) ** 2))) for x in (got, once)]
    print(f"rms {rms[0]:.3e}, rounded once {rms[1]:.3e}, ratio {rms[0] / rms[1]:.4f}")
    assert rms[0] <= 1.03 * rms[1]


@pytest.mark.parametrize("spread", [1.0, 1.64, 2.5])
def test_sinks_cost_a_model_no_precision(spread):
    """The exact layer of test_gpu_attn_precision, with a window that nothing has passed yet: with sinks and without, the
    prompts see the same keys."""
    ax = _ax()
    w, parts = _model(spread)
    ids = np.random.default_rng(6).integers(0, V, (N, S)).astype(np.int32)
    ref = _exact(ids, *parts)
    rms = []
    for sinks in (4, 0):
        m = create(dict(SHAPE, window=2 * S, sinks=sinks), w, max_batch=8, max_context=S, max_prefill_tokens=8 * S, fp16=True)
        try:
            lg = np.concatenate([run_prefill(m, ids[i:i + 8], ax.AXON_LOGITS_LAST, V)[0] for i in range(0, N, 8)]).reshape(N, V)
            assert ax.axon_check_device(m)[0] == 0
        finally:
            ax.axon_free(m)
        rms.append(float(np.sqrt(np.mean((lg - ref) ** 2))))
    print(f"spread {spread}: rms {rms[0]:.3e} with sinks, {rms[1]:.3e} without, ratio {rms[0] / rms[1]:.4f}")
    # (the bound of test_gpu_attn_precision: two errors of equal expectation over 1,024 groups)
    assert rms[0] <= 1.008 * rms[1]
