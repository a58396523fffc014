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
                         max_prefill_tokens=128)
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

def test_rows_past_the_tokens_are_left_as_they_are():
    """A step and a piece for the first rows only: an ended row takes no blocks, a waiting one keeps its own."""
    shape = dict(TINY, window=64, sinks=4)
    ax = _ax()
    m, seqs, w = seqs_of(shape, 3, 40)
    try:
        text = [si.make_ids(1, n, shape["V"], seed=n)[0] for n in (30, 21, 17)]
        seqs.extend(ints(np.concatenate(text)), [30, 21, 17])
        seqs.release(ints([2]))
        held = seqs.table[1:].clone()
        logits = torch.empty(1, shape["V"], device="cuda")
        for i in range(20):
            text[0] = np.append(text[0], i)
            seqs.step(ints([i]), logits=logits)
        seqs.check()
        assert seqs.lengths() == [50, 21, 0]
        assert torch.equal(seqs.table[1:], held) and int((held[1] >= 0).sum()) == 0
        assert seqs.blocks_in_use() == 4 + 2
        assert np.abs(logits[0].cpu().numpy() - last_logits(shape, w, text[0])).max() <= tiny_tol("bf16")
        # the other rows go on from there
        seqs.extend(ints([7, 8, 9]), [1, 2], logits=torch.empty(2, shape["V"], device="cuda"))
        both = torch.empty(2, shape["V"], device="cuda")
        seqs.step(ints([3, 4]), logits=both)
        seqs.check()
        assert seqs.lengths() == [52, 24, 0]
        for b, tail in ((0, [7, 3]), (1, [8, 9, 4])):
            want = last_logits(shape, w, np.append(text[b], tail))
            assert np.abs(both[b].cpu().numpy() - want).max() <= tiny_tol("bf16")
        with pytest.raises(ValueError):
            seqs.step(ints([1, 2, 3, 4]))
        with pytest.raises(ValueError):
            seqs.extend(ints([]), [])
    finally:
        ax.axon_free(m)
