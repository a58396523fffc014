"""Refusals of axon_sample that need no GPU."""
import pytest

torch = pytest.importorskip("torch")

FAKE = 1 << 20  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def ax():
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


def sample(ax, **change):
    a = dict(logits=FAKE, stride=1000, precision=ax.AXON_FP32_DEBUG, B=2, V=1000, temp=None, k=None, p=None, m=None, u=FAKE,
             tokens=FAKE, prob=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return ax.lib().axon_sample(*a.values())


@pytest.mark.parametrize("change", [dict(logits=None), dict(logits=FAKE + 2), dict(u=None), dict(tokens=None), dict(B=0), dict(V=0),
                                    dict(stride=999), dict(stride=-1000), dict(precision=3), dict(precision=-1),
                                    dict(precision=0, logits=FAKE + 1)], ids=str)
def test_refuses(ax, change):
    assert sample(ax, **change) == ax.AXON_ERR_INVALID_ARG


def test_limits(ax):
    assert sample(ax, V=524289, stride=524289) == ax.AXON_ERR_UNSUPPORTED
    assert sample(ax, B=(1 << 24) + 1) == ax.AXON_ERR_UNSUPPORTED


def test_the_binding_refuses(ax):
    x, u, t = torch.zeros(2, 10), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        ax.axon_sample(x, u, t)  # host memory
    with pytest.raises(TypeError):
        ax.axon_sample(x.double(), u, t)
    with pytest.raises(TypeError):
        ax.axon_sample(x.view(-1), u, t)
