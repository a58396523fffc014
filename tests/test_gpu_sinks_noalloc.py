"""The allocation-free decode step of a model with attention sinks: its attention needs none of the fixed merge slots, whose
number limits the other models' batches."""
import numpy as np
import pytest

import synth_inputs as si
from helpers import create, gpu_weights
from test_gpu_parity import TINY, _ax

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SINK = dict(TINY, D=512, H=8, G=8, window=24, sinks=4)


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()


@pytest.mark.parametrize("B", [3, 33, 64])
def test_batches_of_more_than_256_rows_and_heads(B):
    ax = _ax()
    S = 40
    m = create(SINK, gpu_weights(SINK), max_batch=B, max_context=64, max_prefill_tokens=B * S)
    try:
        tok = torch.empty(B, dtype=torch.int32, device="cuda")
        ax.axon_prefill(m, torch.from_numpy(si.make_ids(B, S, SINK["V"], seed=7)).cuda(), next_tokens=tok)
        out = []
        for step in (ax.axon_decode_step, ax.axon_decode_step_noalloc):
            ctx = torch.full((B,), S, dtype=torch.int32, device="cuda")
            logits = torch.full((B, SINK["V"]), float("nan"), device="cuda")
            step(m, tok, ctx, logits=logits, next_tokens=torch.empty_like(tok))
            out.append(logits.cpu().numpy())
        assert ax.axon_check_device(m)[0] == 0
        assert np.isfinite(out[0]).all() and np.array_equal(out[0], out[1])
    finally:
        ax.axon_free(m)
