"""Refusals of the operators on a paged key/value cache that need no GPU: the C
entry points check what the host can see before any device call, the binding checks
types, shapes and layouts."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

FAKE = 1 << 20  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def ax():
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


def cache(ax, **change):
    f = dict(k_pool=FAKE, v_pool=FAKE, num_layers=2, num_blocks=64, num_kv_heads=2, block_size=16, head_dim=64,
             precision=ax.AXON_BF16)
    f.update(change)
    return ax.axon_kv_cache(**f)


def decode(ax, c=None, **change):
    a = dict(layer=0, q=FAKE, qr=512, qh=64, B=2, H=8, ctx=FAKE, table=FAKE, per=4, window=0, sinks=0, scale=0.0, o=FAKE,
             orow=512, oh=64, lse=None, work=FAKE, bytes=1 << 40, err=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return ax.lib().axon_attn_decode(ctypes.byref(c or cache(ax)), *a.values())


def prefill(ax, c=None, **change):
    a = dict(layer=0, q=FAKE, qr=512, qh=64, B=2, T=20, H=8, cu=FAKE, ctx=FAKE, longest=15, table=FAKE, per=4, window=0,
             sinks=0, scale=0.0, o=FAKE, orow=512, oh=64, err=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return ax.lib().axon_attn_prefill(ctypes.byref(c or cache(ax)), *a.values())


COMMON = [dict(layer=2), dict(layer=-1), dict(q=None), dict(o=None), dict(q=FAKE + 8), dict(o=FAKE + 2), dict(H=7), dict(H=0),
          dict(per=0), dict(window=-1), dict(sinks=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
          dict(ctx=None), dict(B=0), dict(qr=0), dict(qh=32), dict(qr=516), dict(orow=60), dict(oh=0),
          dict(table=None, per=33)]


@pytest.mark.parametrize("change", COMMON + [dict(work=None), dict(work=FAKE + 4)], ids=str)
def test_decode_refuses(ax, change):
    assert decode(ax, **change) == ax.AXON_ERR_INVALID_ARG


@pytest.mark.parametrize("change", COMMON + [dict(cu=None), dict(T=0), dict(longest=0), dict(longest=21)], ids=str)
def test_prefill_refuses(ax, change):
    assert prefill(ax, **change) == ax.AXON_ERR_INVALID_ARG


@pytest.mark.parametrize("change,want", [
    (dict(k_pool=None), 1), (dict(v_pool=FAKE + 2), 1), (dict(num_layers=0), 1), (dict(num_blocks=0), 1),
    (dict(num_kv_heads=0), 1), (dict(precision=9), 1), (dict(block_size=32), 4), (dict(head_dim=96), 4),
    (dict(precision=1), 4)], ids=str)
def test_caches_that_the_attention_refuses(ax, change, want):
    assert decode(ax, cache(ax, **change)) == want
    assert prefill(ax, cache(ax, **change)) == want


def test_limits(ax):
    assert decode(ax, B=2049) == ax.AXON_ERR_UNSUPPORTED
    assert decode(ax, B=2048, per=1 << 20) == ax.AXON_ERR_UNSUPPORTED  # 2^32 pages
    assert decode(ax, H=34, qr=34 * 64, orow=34 * 64) == ax.AXON_ERR_UNSUPPORTED  # 17 query heads per kv head
    assert prefill(ax, H=34, qr=34 * 64, orow=34 * 64) == ax.AXON_ERR_UNSUPPORTED
    assert ax.lib().axon_attn_decode(None, 0, FAKE, 64, 64, 1, 1, FAKE, FAKE, 1, 0, 0, 0.0, FAKE, 64, 64, None, FAKE, 1 << 40,
                                     None, None) == ax.AXON_ERR_INVALID_ARG


def seqs(ax, **change):
    f = dict(block_table=FAKE, context_lens=FAKE, refs=FAKE, max_seqs=4, blocks_per_seq=8)
    f.update(change)
    return ax.axon_kv_seqs(**f)


def test_block_operators_refuse(ax):
    L, bad = ax.lib(), ax.AXON_ERR_INVALID_ARG
    c, s = cache(ax), seqs(ax)
    n = ctypes.c_int64()
    assert L.axon_kv_workspace(ctypes.byref(c), ctypes.byref(s), ctypes.byref(n)) == 0 and n.value > 0
    C, S, W = ctypes.byref(c), ctypes.byref(s), n.value
    assert L.axon_kv_fork(C, S, FAKE, FAKE, 5, FAKE, W, None, None) == bad  # more entries than rows
    assert L.axon_kv_fork(C, S, None, FAKE, 2, FAKE, W, None, None) == bad
    assert L.axon_kv_fork(C, S, FAKE, FAKE, -1, FAKE, W, None, None) == bad
    assert L.axon_kv_fork(C, S, FAKE, FAKE, 2, FAKE, W - 4, None, None) == bad
    assert L.axon_kv_fork(C, S, FAKE, FAKE, 2, FAKE + 4, W, None, None) == bad
    assert L.axon_kv_fork(C, S, FAKE, FAKE, 2, FAKE, -1, None, None) == bad
    assert L.axon_kv_fork(C, None, FAKE, FAKE, 2, FAKE, W, None, None) == bad
    assert L.axon_kv_reserve(C, S, FAKE, None, 2, FAKE, W, None, None) == bad
    assert L.axon_kv_reserve(C, S, FAKE, FAKE, 2, None, W, None, None) == bad
    assert L.axon_kv_release(C, S, FAKE, 5, 0, 0, None, None) == bad
    assert L.axon_kv_release(C, S, FAKE, 2, -1, 0, None, None) == bad
    assert L.axon_kv_release(C, S, FAKE, 2, 16, -1, None, None) == bad
    assert L.axon_kv_compact(C, S, None, None, None, W, None, None) == bad
    assert L.axon_kv_copy_blocks(C, None, FAKE, 2, None, None) == bad
    assert L.axon_kv_copy_blocks(C, FAKE, FAKE, -1, None, None) == bad
    assert L.axon_check_error(None, None, None) == bad
    assert L.axon_kv_cache_get(None, C) == bad
    for change in (dict(block_table=None), dict(context_lens=None), dict(refs=None), dict(max_seqs=0), dict(blocks_per_seq=0)):
        assert L.axon_kv_release(C, ctypes.byref(seqs(ax, **change)), FAKE, 1, 0, 0, None, None) == bad
    assert L.axon_kv_release(C, ctypes.byref(seqs(ax, max_seqs=8193)), FAKE, 1, 0, 0, None, None) == ax.AXON_ERR_UNSUPPORTED
    assert L.axon_kv_release(C, ctypes.byref(seqs(ax, max_seqs=8192, blocks_per_seq=1 << 18)), FAKE, 1, 0, 0, None, None) == \
        ax.AXON_ERR_UNSUPPORTED
    # nothing to do
    assert L.axon_kv_fork(C, S, None, None, 0, FAKE, W, None, None) == 0
    assert L.axon_kv_release(C, S, None, 0, 0, 0, None, None) == 0


def test_the_binding_refuses_host_and_mistyped_tensors(ax):
    k = torch.zeros(1, 4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        ax.make_kv_cache(k, k)  # host memory
    with pytest.raises(TypeError):
        ax.make_kv_cache(k.double(), k.double())
    with pytest.raises(TypeError):
        ax.make_kv_seqs(torch.zeros(2, 4, dtype=torch.int64), torch.zeros(2), torch.zeros(4))
