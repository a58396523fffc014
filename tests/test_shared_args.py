"""Refusals of axon_attn_shared that need no GPU."""
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


def shared(ax, c=None, cache={}, **change):
    f = dict(k_pool=FAKE, v_pool=FAKE, num_layers=2, num_blocks=64, num_kv_heads=2, block_size=16, head_dim=64,
             precision=ax.AXON_BF16)
    f.update(cache)
    a = dict(layer=0, q=FAKE, qr=512, qh=64, B=2, H=8, ctx=FAKE, table=FAKE, per=4, offsets=FAKE, prefix=FAKE, N=1, window=0,
             sinks=0, scale=0.0, o=FAKE, orow=512, oh=64, lse=None, work=FAKE, bytes=1 << 40, err=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return ax.lib().axon_attn_shared(ctypes.byref(ax.axon_kv_cache(**f)), *a.values())


@pytest.mark.parametrize("change", [
    dict(layer=2), dict(q=None), dict(o=None), dict(q=FAKE + 8), dict(o=FAKE + 2), dict(H=7), dict(per=0), dict(window=-1),
    dict(sinks=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(ctx=None), dict(B=0), dict(qr=0), dict(qh=32), dict(qr=516),
    dict(oh=0), dict(table=None), dict(offsets=None), dict(prefix=None), dict(N=0), dict(N=-1), dict(work=None),
    dict(work=FAKE + 4)], ids=str)
def test_refuses(ax, change):
    assert shared(ax, **change) == ax.AXON_ERR_INVALID_ARG


def test_limits(ax):
    assert shared(ax, N=1025) == ax.AXON_ERR_UNSUPPORTED
    assert shared(ax, B=2049) == ax.AXON_ERR_UNSUPPORTED
    assert shared(ax, H=34, qr=34 * 64, orow=34 * 64) == ax.AXON_ERR_UNSUPPORTED
    assert shared(ax, cache=dict(precision=1)) == ax.AXON_ERR_UNSUPPORTED
    assert shared(ax, cache=dict(head_dim=96)) == ax.AXON_ERR_UNSUPPORTED
    assert ax.lib().axon_attn_shared_workspace(None, 8, 2, None) == ax.AXON_ERR_INVALID_ARG
