"""Refusals of axon_kv_append and axon_rope_table that need no GPU."""
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


def append(ax, c=None, **change):
    a = dict(layer=0, q=FAKE, qr=512, qh=64, k=FAKE, kr=128, kh=64, v=FAKE, vr=128, vh=64, B=2, T=20, H=8, cu=FAKE, ctx=FAKE,
             table=FAKE, per=4, rope=FAKE, positions=64, rotary=64, layout=0, o=FAKE + 4096, orow=512, oh=64, err=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return ax.lib().axon_kv_append(ctypes.byref(c or cache(ax)), *a.values())


@pytest.mark.parametrize("change", [
    dict(layer=2), dict(layer=-1), dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(q=FAKE + 8),
    dict(o=FAKE + 8), dict(q=None), dict(o=None), dict(q=None, o=None), dict(H=0), dict(H=-1), dict(B=0), dict(T=0),
    dict(cu=None), dict(ctx=None), dict(per=0), dict(per=1 << 27), dict(table=None, per=33), dict(kr=60), dict(kh=32),
    dict(vr=132), dict(vh=68), dict(qr=0), dict(oh=0), dict(rope=None), dict(rope=FAKE + 8), dict(rotary=0), dict(rotary=80),
    dict(rotary=-16), dict(positions=0), dict(layout=2), dict(o=FAKE, orow=1024)], ids=str)
def test_refuses(ax, change):
    assert append(ax, **change) == ax.AXON_ERR_INVALID_ARG


def test_limits(ax):
    assert append(ax, rotary=40) == ax.AXON_ERR_UNSUPPORTED  # not a multiple of 16
    assert append(ax, cache(ax, head_dim=96)) == ax.AXON_ERR_UNSUPPORTED
    assert append(ax, cache(ax, precision=9)) == ax.AXON_ERR_INVALID_ARG


@pytest.mark.parametrize("a,want", [
    ((None, 64, 64, 1e4, 0.0, 1.0, 4.0, 8192), 1), ((FAKE + 4, 64, 64, 1e4, 0.0, 1.0, 4.0, 8192), 1),
    ((FAKE, 0, 64, 1e4, 0.0, 1.0, 4.0, 8192), 1), ((FAKE, 64, 0, 1e4, 0.0, 1.0, 4.0, 8192), 1),
    ((FAKE, 64, 64, 0.0, 0.0, 1.0, 4.0, 8192), 1), ((FAKE, 64, 64, float("nan"), 0.0, 1.0, 4.0, 8192), 1),
    ((FAKE, 64, 64, 1e4, -1.0, 1.0, 4.0, 8192), 1), ((FAKE, 64, 64, 1e4, 8.0, 4.0, 1.0, 8192), 1),
    ((FAKE, 64, 64, 1e4, 8.0, 1.0, 4.0, 0), 1), ((FAKE, 64, 24, 1e4, 0.0, 1.0, 4.0, 8192), 4),
    ((FAKE, 64, 144, 1e4, 0.0, 1.0, 4.0, 8192), 4)], ids=str)
def test_the_table_refuses(ax, a, want):
    assert ax.lib().axon_rope_table(*a, None) == want
