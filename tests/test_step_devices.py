"""axon_kv_append, axon_attn_shared, axon_sample and axon_rope_table with operands on another device than the cache's (or the
logits'), in host memory, or under another current device: the binding refuses the call before anything is launched. As
in test_kv_devices.py, nothing here touches a GPU."""
import pytest

torch = pytest.importorskip("torch")
from test_kv_devices import Tensor as Dense, ax  # noqa: E402, F401


class Tensor(Dense):
    def stride(self, dim=None):
        return super().stride() if dim is None else super().stride()[dim]



F32, I32, BF16 = torch.float32, torch.int32, torch.bfloat16
OPERANDS = dict(k=((1, 8, 2, 16, 64), BF16), v=((1, 8, 2, 16, 64), BF16), q=((3, 4, 64), BF16), out=((3, 4, 64), BF16),
                new_k=((3, 2, 64), BF16), new_v=((3, 2, 64), BF16), ctx=((3,), I32), bt=((3, 2), I32), cu=((4,), I32),
                lse=((3, 4), F32), err=((1,), I32), work=((1 << 20,), torch.uint8), offsets=((3,), I32), prefix=((2,), I32),
                rope=((32, 32, 2), F32), x=((3, 50), BF16), u=((3,), F32), tok=((3,), I32), temp=((3,), F32), top_k=((3,), I32),
                top_p=((3,), F32), min_p=((3,), F32), prob=((3,), F32))
READS = {"append": ["v", "q", "out", "new_k", "new_v", "ctx", "bt", "cu", "rope", "err"],
         "shared": ["v", "q", "out", "ctx", "bt", "offsets", "prefix", "lse", "work", "err"],
         "sample": ["u", "tok", "temp", "top_k", "top_p", "min_p", "prob"]}
NAMES = {"append": "axon_kv_append", "shared": "axon_attn_shared", "sample": "axon_sample"}


def call(ax, op, device=0, **change):  # noqa: F811
    t = type("Use", (), {n: Tensor(*OPERANDS[n], device) for n in OPERANDS} | change)
    if op == "sample":
        return ax.axon_sample(t.x, t.u, t.tok, t.temp, t.top_k, t.top_p, t.min_p, t.prob)
    cache = ax.make_kv_cache(t.k, t.v)
    if op == "append":
        return ax.axon_kv_append(cache, 0, t.new_k, t.new_v, t.ctx, block_table=t.bt, cu_seqlens=t.cu, rope=t.rope, q=t.q,
                                 q_out=t.out, err=t.err)
    return ax.axon_attn_shared(cache, 0, t.q, t.ctx, t.offsets, t.prefix, t.out, t.work, t.bt, lse=t.lse, err=t.err)


@pytest.mark.parametrize("op", sorted(READS))
def test_operands_of_one_device_are_taken(ax, op):  # noqa: F811
    call(ax, op)
    assert ax._calls == [NAMES[op]]


@pytest.mark.parametrize("device", [1, -1])
@pytest.mark.parametrize("op,name", [(op, n) for op in sorted(READS) for n in READS[op]])
def test_an_operand_elsewhere_is_refused(ax, op, name, device):  # noqa: F811
    with pytest.raises(TypeError):
        call(ax, op, **{name: Tensor(*OPERANDS[name], device)})
    assert not ax._calls


@pytest.mark.parametrize("op", sorted(READS))
def test_another_current_device_is_refused(ax, op):  # noqa: F811
    with pytest.raises((TypeError, ValueError)):
        call(ax, op, device=1)
    assert not ax._calls


def test_streams_and_tables_of_another_device_are_refused(ax, monkeypatch):  # noqa: F811
    class Stream:
        cuda_stream, device_index = 77, 1

    with pytest.raises((TypeError, ValueError)):
        ax.axon_sample(*(Tensor(*OPERANDS[n]) for n in ("x", "u", "tok")), stream=Stream())
    monkeypatch.setattr(torch, "empty", lambda *shape, device, **k: Tensor(shape, F32, torch.device(device).index))
    ax.axon_rope_table(32, 64, 1e4)
    with pytest.raises((TypeError, ValueError)):
        ax.axon_rope_table(32, 64, 1e4, device="cuda:1")
    assert ax._calls == ["axon_rope_table"]


def test_logits_in_host_memory_are_refused(ax):  # noqa: F811
    with pytest.raises(TypeError):
        call(ax, "sample", x=Tensor(*OPERANDS["x"], -1))
    assert not ax._calls


def test_workspaces_are_made_where_the_cache_is(ax, monkeypatch):  # noqa: F811
    made = []
    monkeypatch.setattr(torch, "zeros", lambda *a, device, **k: made.append(torch.device(device)))
    monkeypatch.setattr(ax, "_current_device", lambda: 1, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    ax.make_shared_workspace(ax.make_kv_cache(Tensor(*OPERANDS["k"], 1), Tensor(*OPERANDS["v"], 1)), 3, 4)
    assert made == [torch.device("cuda", 1)]
