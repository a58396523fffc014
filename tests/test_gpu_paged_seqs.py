"""Sequences on managed cache blocks (paged.PagedSeqs) where the pool is small: prompts fed in pieces, rows that
are left as they are by a step, and windows without sinks."""
import numpy as np
import pytest

import synth_inputs as si
from helpers import gpu_weights, oracle_for, tiny_tol
from test_gpu_parity import TINY, _ax

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()


def seqs_of(shape, rows, blocks, max_context=512, max_batch=None):
    from paper_2608_19889_gb300 import paged
    ax = _ax()
    w = gpu_weights(shape)
    cfg = ax.make_config(shape, max_batch or rows, max_context, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=blocks,
                         max_prefill_tokens=64)
    m = ax.axon_model_create(cfg, w)
    return m, paged.PagedSeqs(m, cfg, rows), w


def ints(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()


def last_logits(shape, w, text):
    o = oracle_for(shape, w)
    ids = np.asarray([text], dtype=np.int32)
    return o.prefill(ids, o.new_contiguous_cache(1, 512), last_only=True)[0, -1]


@pytest.mark.parametrize("window,sinks", [(40, 4), (40, 0), (33, 20)])
def test_a_long_prompt_in_pieces_needs_no_more_than_its_window(window, sinks):
    """300 tokens of two rows, 32 at a time: a piece and its window reach 71 tokens, 6 blocks at most, and the sinks 2."""
    shape = dict(TINY, window=window, sinks=sinks)
    ax = _ax()
    m, seqs, w = seqs_of(shape, 2, 16)
    try:
        text = [si.make_ids(1, 300, shape["V"], seed=5 + b)[0] for b in range(2)]
        for at in range(0, 300, 32):
            n = min(32, 300 - at)
            logits = torch.empty(2, shape["V"], device="cuda")
            seqs.extend(ints(np.concatenate([t[at:at + n] for t in text])), [n, n], logits=logits)
            seqs.check()
            assert seqs.blocks_in_use() <= 16
        for b in range(2):
            assert np.abs(logits[b].cpu().numpy() - last_logits(shape, w, text[b])).max() <= tiny_tol("bf16")
        for i in range(40):  # and on
            tok = np.asarray([i + 1, 2 * i + 1], dtype=np.int32)
            text = [np.append(t, tok[b]) for b, t in enumerate(text)]
            seqs.step(ints(tok), logits=logits)
        seqs.check()
        for b in range(2):
            assert np.abs(logits[b].cpu().numpy() - last_logits(shape, w, text[b])).max() <= tiny_tol("bf16")
    finally:
        ax.axon_free(m)
