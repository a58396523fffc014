"""PagedSeqs.sample refuses operands of axon_sample before it takes the step. Nothing here touches a GPU."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_19889_gb300 import paged  # noqa: E402
from test_step_devices import Tensor, ax  # noqa: E402, F401

F32, I32 = torch.float32, torch.int32
GOOD = dict(u=((3,), F32), next_tokens=((3,), I32), temperature=((3,), F32), top_k=((3,), I32), top_p=((3,), F32), min_p=((3,), F32),
            prob=((3,), F32))


@pytest.fixture
def seqs(ax, monkeypatch):  # noqa: F811
    s = paged.PagedSeqs.__new__(paged.PagedSeqs)
    s.rows, s.vocabulary, s.logits, s.steps, s.all = 4, 100, None, [], Tensor((4,), I32)
    s.cache = ax.make_kv_cache(*(Tensor((1, 8, 2, 16, 64), torch.bfloat16) for _ in range(2)))
    monkeypatch.setattr(s, "step", lambda tokens, logits: s.steps.append(tokens.numel()), raising=False)

    class Logits(Tensor):
        def __getitem__(self, key):
            return Logits((3, 100), F32, self.index)
    monkeypatch.setattr(torch, "empty", lambda *shape, device, **k: Logits(shape, F32, torch.device(device).index or 0))
    return s


def sample(s, **change):
    t = {n: Tensor(*v) for n, v in GOOD.items()} | change
    s.sample(Tensor((3,), I32), t.pop("u"), t.pop("next_tokens"), **t)


def test_good_operands(ax, seqs):  # noqa: F811
    sample(seqs)
    sample(seqs, temperature=None, top_k=None, top_p=None, min_p=None, prob=None)
    assert seqs.steps == [3, 3] and ax._calls == ["axon_sample"] * 2


@pytest.mark.parametrize("name", sorted(GOOD))
def test_bad_ones_take_no_step(ax, seqs, name):  # noqa: F811
    shape, dtype = GOOD[name]
    for bad in (Tensor((4,), dtype), Tensor(shape, torch.float64), Tensor(shape, dtype, 1), Tensor(shape, dtype, -1)):
        with pytest.raises(TypeError):
            sample(seqs, **{name: bad})
    assert not seqs.steps and not ax._calls


@pytest.mark.parametrize("name", ["u", "next_tokens"])
def test_what_has_to_be_there(ax, seqs, name):  # noqa: F811
    with pytest.raises(TypeError):
        sample(seqs, **{name: None})
    assert not seqs.steps and not ax._calls


def test_logits_are_where_the_rows_are(ax, seqs, monkeypatch):  # noqa: F811
    """Not on the device that happens to be current with the first call, where every later one would be refused."""
    made = []
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *shape, device, **k: made.append(torch.device(device)) or empty(*shape, device=device))
    sample(seqs)
    assert made == [torch.device("cuda", 0)]
