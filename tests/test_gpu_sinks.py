"""A model whose sliding window keeps its first tokens visible (sink_tokens), against
the oracle: prompts, chunks after a past, decode steps, contiguous and paged, both 16-bit
modes; block management under it, and the streaming example."""
import os
import sys

import numpy as np
import pytest

import synth_inputs as si
from helpers import create, gpu_weights, oracle_for, tiny_tol
from test_gpu_parity import TINY, TINY128, _ax, check, decode_steps, oracle_decode, run_prefill
from test_gpu_varlen import _case

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SINK = dict(TINY, window=24, sinks=4)
SINK128 = dict(TINY128, window=40, sinks=19)


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()


@pytest.mark.parametrize("prec", ["bf16", "fp16"])
@pytest.mark.parametrize("shape,B,S,max_ctx", [(SINK, 2, 100, 128), (SINK128, 3, 70, 128), (SINK, 2, 20, 128), (SINK, 1, 1, 64),
                                               (dict(TINY, window=200, sinks=1), 2, 600, 640)])
def test_sinks_prefill_all_positions_and_decode(shape, B, S, max_ctx, prec):
    ax = _ax()
    w = gpu_weights(shape)
    m = create(shape, w, max_batch=B, max_context=max_ctx, max_prefill_tokens=B * S, fp16=prec == "fp16")
    try:
        ids = si.make_ids(B, S, shape["V"], seed=31)
        lg, nxt = run_prefill(m, ids, ax.AXON_LOGITS_ALL, shape["V"])
        o = oracle_for(shape, w)
        cache = o.new_contiguous_cache(B, max_ctx)
        check(lg, o.prefill(ids, cache), tol=tiny_tol(prec), what=f"sinks {shape['sinks']} prefill S={S}")
        dl, fed = decode_steps(m, nxt, [S] * B, 10, shape["V"])
        check(dl, oracle_decode(o, cache, fed, [S] * B), tol=tiny_tol(prec), what="sinks decode")
        assert ax.axon_check_device(m)[0] == 0
    finally:
        ax.axon_free(m)


@pytest.mark.parametrize("layout", ["contiguous", "paged"])
def test_sinks_varlen_chunks_after_a_long_past(layout):
    _case(SINK, layout, "bf16", first=[90, 40, 1], second=[30, 1, 64])


def test_sinks_are_seen():
    """The same window without sinks gives other logits past it, and the same ones before."""
    ax = _ax()
    w = gpu_weights(SINK)
    out = []
    for shape in (SINK, dict(SINK, sinks=0)):
        m = create(shape, w, max_batch=1, max_context=128)
        lg, _ = run_prefill(m, si.make_ids(1, 60, SINK["V"], seed=3), ax.AXON_LOGITS_ALL, SINK["V"])
        out.append(np.asarray(lg))
        ax.axon_free(m)
    assert np.abs(out[0][0, :24] - out[1][0, :24]).max() < 2 * tiny_tol("bf16")
    assert np.abs(out[0][0, 28:] - out[1][0, 28:]).max() > 2 * tiny_tol("bf16")


@pytest.mark.parametrize("change,want", [(dict(sink_tokens=-1), 1), (dict(sink_tokens=4, sliding_window=0), 1),
                                         (dict(sink_tokens=4, precision=1), 4)])
def test_sinks_refused(change, want):
    import ctypes
    ax = _ax()
    cfg = ax.make_config(SINK, 1, 64)
    for k, v in change.items():
        setattr(cfg, k, v)
    out = ctypes.c_void_p()
    assert ax.lib().axon_model_create(ctypes.byref(cfg), None, 0, None, ctypes.byref(out)) == want


@pytest.mark.parametrize("prec", ["bf16", "fp16"])
def test_managed_blocks_give_what_a_roomy_cache_gives(prec):
    """Forked, released, reserved and compacted blocks against the oracle's steps on a cache of its own."""
    from paper_2608_19889_gb300 import paged
    ax = _ax()
    shape, B, S, steps = dict(SINK, window=40), 3, 45, 70
    w = gpu_weights(shape)
    cfg = ax.make_config(shape, B, 256, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=20, max_prefill_tokens=64,
                         precision=ax.AXON_FP16 if prec == "fp16" else ax.AXON_BF16)
    m = ax.axon_model_create(cfg, w)
    try:
        seqs = paged.PagedSeqs(m, cfg, B)
        V = shape["V"]
        rng = np.random.default_rng(7)
        prompt = si.make_ids(1, S, V, seed=5)[0]
        ids = torch.from_numpy(np.concatenate([prompt, [1, 2]]).astype(np.int32)).cuda()
        seqs.extend(ids, [S, 1, 1])
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        seqs.fork(ints(0, 0), ints(1, 2))
        text = [list(prompt) for _ in range(B)]
        fed = rng.integers(0, V, (steps, B)).astype(np.int32)
        got, rows = [], []
        for i in range(steps):
            if i == 30:  # row 1 goes on as row 2 stands
                seqs.fork(ints(2), ints(1))
                text[1] = list(text[2])
            if i % 16 == 7:
                seqs.compact()
            logits = torch.empty(B, V, device="cuda")
            for b in range(B):
                text[b].append(fed[i, b])
            seqs.step(torch.from_numpy(fed[i]).cuda(), logits=logits)
            if i in (0, 29, 30, steps - 1):
                got.append(logits.cpu().numpy())
                rows.append([list(t) for t in text])
        seqs.check()
        assert seqs.blocks_in_use() < B * (-(-len(text[0]) // 16))
        assert torch.equal(torch.bincount(seqs.table[seqs.table >= 0], minlength=20).int(), seqs.refs)
        o = oracle_for(shape, w)
        for logits, texts in zip(got, rows):
            for b in range(B):
                ref = o.prefill(np.asarray([texts[b]], dtype=np.int32), o.new_contiguous_cache(1, 256), last_only=True)[0, -1]
                # a step's logits and its oracle's: the tolerance of the tiny shapes
                assert np.abs(logits[b] - ref).max() <= tiny_tol(prec)
    finally:
        ax.axon_free(m)


def test_more_sinks_than_positions_are_no_window():
    """Sinks that cover the context: the plain causal mask, whatever the window."""
    ax = _ax()
    w = gpu_weights(SINK)
    out = []
    for shape in (dict(SINK, sinks=2 ** 31 - 1), dict(SINK, window=2 ** 31 - 1)):
        m = create(shape, w, max_batch=1, max_context=128)
        out.append(run_prefill(m, si.make_ids(1, 90, SINK["V"], seed=3), ax.AXON_LOGITS_ALL, SINK["V"])[0])
        ax.axon_free(m)
    assert np.array_equal(out[0], out[1])


def test_paged_seqs_refuses():
    from paper_2608_19889_gb300 import paged
    ax = _ax()
    with pytest.raises(ValueError):
        paged.PagedSeqs(None, ax.make_config(SINK, 2, 64), 1)
    with pytest.raises(ValueError):
        paged.PagedSeqs(None, ax.make_config(SINK, 2, 64, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=4), 3)


def test_a_pool_that_is_too_small_is_reported():
    from paper_2608_19889_gb300 import paged
    ax = _ax()
    cfg = ax.make_config(SINK, 1, 256, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=2, max_prefill_tokens=64)
    m = ax.axon_model_create(cfg, gpu_weights(SINK))
    try:
        seqs = paged.PagedSeqs(m, cfg, 1)
        seqs.extend(torch.zeros(40, dtype=torch.int32, device="cuda"), [40])
        with pytest.raises(ax.AxonError):
            seqs.check()
    finally:
        ax.axon_free(m)


def test_streaming_example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import streaming
    lines = []
    out, most = streaming.generate(steps=200, say=lines.append)
    assert out.shape == (201, streaming.SAMPLES) and most < streaming.POOL
    assert int(out.min()) >= 0 and int(out.max()) < streaming.SHAPE["V"]
    assert torch.equal(out[101, 0], out[101, 3])  # the fork in the middle starts from sample 0's state
    assert len(lines) == 4
