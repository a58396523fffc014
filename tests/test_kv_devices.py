"""Operands on another device than the cache's, in host memory, or under another current device: the binding refuses
the call before anything is launched. Nothing here touches a GPU: the tensors are stand-ins with the attributes that the
binding reads, and the library is one that counts its calls."""
import pytest

torch = pytest.importorskip("torch")


class Tensor:
    """A dense tensor as the binding sees it; device -1: host memory."""

    def __init__(self, shape, dtype, device=0, at=1 << 20):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at
        self.index = device
        self.is_cuda = device >= 0
        self.device = torch.device("cuda", device) if device >= 0 else torch.device("cpu")
        self.nbytes = self.numel() * 2

    def get_device(self):
        return self.index

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self):
        s, out = 1, []
        for n in reversed(self.shape):
            out.insert(0, s)
            s *= n
        return tuple(out)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if not name.startswith("axon_"):
            raise AttributeError(name)
        return lambda *a: self.calls.append(name) or 0


@pytest.fixture
def ax(monkeypatch):
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    ax.lib()
    library = Library()
    monkeypatch.setattr(ax, "_lib", library)
    monkeypatch.setattr(ax, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(ax, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(ax, "_calls", library.calls, raising=False)
    return ax


def i32(*shape, device=0):
    return Tensor(shape, torch.int32, device)


def half(*shape, device=0):
    return Tensor(shape, torch.bfloat16, device)


def calls(ax, device=0, **change):
    """Each operator's call on operands of `device`; change: operands of another one, by name."""
    t = dict(k=half(1, 8, 2, 16, 64, device=device), v=half(1, 8, 2, 16, 64, device=device), q=half(3, 4, 64, device=device),
             out=half(3, 4, 64, device=device), ctx=i32(3, device=device), bt=i32(3, 2, device=device),
             cu=i32(4, device=device), lse=Tensor((3, 4), torch.float32, device), err=i32(1, device=device),
             work=Tensor((1 << 20,), torch.uint8, device), table=i32(3, 2, device=device), lens=i32(3, device=device),
             refs=i32(8, device=device), a=i32(2, device=device), b=i32(2, device=device), moved=i32(8, device=device),
             live=i32(1, device=device))
    assert set(change) <= set(t)
    t.update(change)
    use = type("Use", (), t)

    def cache():
        return ax.make_kv_cache(use.k, use.v)

    def seqs():
        return ax.make_kv_seqs(use.table, use.lens, use.refs)

    return {
        "decode": lambda: ax.axon_attn_decode(cache(), 0, use.q, use.ctx, use.out, use.work, block_table=use.bt, lse=use.lse,
                                              err=use.err),
        "prefill": lambda: ax.axon_attn_prefill(cache(), 0, use.q, use.cu, use.ctx, 1, use.out, block_table=use.bt, err=use.err),
        "copy": lambda: ax.axon_kv_copy_blocks(cache(), use.a, use.b, err=use.err),
        "fork": lambda: ax.axon_kv_fork(cache(), seqs(), use.a, use.b, use.work, err=use.err),
        "release": lambda: ax.axon_kv_release(cache(), seqs(), use.a, err=use.err),
        "reserve": lambda: ax.axon_kv_reserve(cache(), seqs(), use.a, use.b, use.work, err=use.err),
        "compact": lambda: ax.axon_kv_compact(cache(), seqs(), use.work, moved=use.moved, live=use.live, err=use.err),
    }


READS = {"decode": ["v", "q", "out", "ctx", "bt", "lse", "err", "work"], "prefill": ["v", "q", "out", "ctx", "bt", "cu", "err"],
         "copy": ["v", "a", "b", "err"], "fork": ["table", "lens", "refs", "a", "b", "err", "work"],
         "release": ["table", "lens", "refs", "a", "err"], "reserve": ["table", "lens", "refs", "a", "b", "err", "work"],
         "compact": ["table", "lens", "refs", "moved", "live", "err", "work"]}


def other(name, device):
    shapes = dict(v=(1, 8, 2, 16, 64), q=(3, 4, 64), out=(3, 4, 64), ctx=(3,), bt=(3, 2), cu=(4,), lse=(3, 4), err=(1,),
                  work=(1 << 20,), table=(3, 2), lens=(3,), refs=(8,), a=(2,), b=(2,), moved=(8,), live=(1,))
    dtype = {"v": torch.bfloat16, "q": torch.bfloat16, "out": torch.bfloat16, "lse": torch.float32,
             "work": torch.uint8}.get(name, torch.int32)
    return Tensor(shapes[name], dtype, device)


@pytest.mark.parametrize("op", sorted(READS))
def test_operands_of_one_device_are_taken(ax, op):
    calls(ax)[op]()
    assert ax._calls == [{"copy": "axon_kv_copy_blocks", "decode": "axon_attn_decode", "prefill": "axon_attn_prefill"}.get(
        op, "axon_kv_" + op)]


@pytest.mark.parametrize("device", [1, -1])
@pytest.mark.parametrize("op,name", [(op, n) for op in sorted(READS) for n in READS[op]])
def test_an_operand_elsewhere_is_refused(ax, op, name, device):
    with pytest.raises(TypeError):
        calls(ax, **{name: other(name, device)})[op]()
    assert not ax._calls


@pytest.mark.parametrize("op", sorted(READS))
def test_another_current_device_is_refused(ax, op):
    """Everything on device 1 while the kernels would go to device 0."""
    with pytest.raises((TypeError, ValueError)):
        calls(ax, device=1)[op]()
    assert not ax._calls


def test_a_stream_of_another_device_is_refused(ax):
    class Stream:
        cuda_stream, device_index = 77, 1

    u = calls(ax)
    u["decode"]()
    c = ax.make_kv_cache(half(1, 8, 2, 16, 64), half(1, 8, 2, 16, 64))
    with pytest.raises((TypeError, ValueError)):
        ax.axon_kv_copy_blocks(c, i32(2), i32(2), stream=Stream())
    assert ax._calls == ["axon_attn_decode"]


def test_workspaces_are_made_where_the_cache_is(ax, monkeypatch):
    made = []
    monkeypatch.setattr(torch, "zeros", lambda *a, device, **k: made.append(torch.device(device)))
    monkeypatch.setattr(torch, "empty", lambda *a, device, **k: made.append(torch.device(device)))
    monkeypatch.setattr(ax, "_current_device", lambda: 1, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    c = ax.make_kv_cache(half(1, 8, 2, 16, 64, device=1), half(1, 8, 2, 16, 64, device=1))
    ax.make_attn_workspace(c, 3, 4)
    ax.make_kv_workspace(c, ax.make_kv_seqs(i32(3, 2, device=1), i32(3, device=1), i32(8, device=1)))
    assert made == [torch.device("cuda", 1)] * 2

def test_a_workspace_that_is_not_dense_is_refused(ax):
    work = Tensor((1 << 20,), torch.uint8)
    work.is_contiguous = lambda: False
    for op in ("decode", "fork", "reserve", "compact"):
        with pytest.raises(TypeError):
            calls(ax, work=work)[op]()
    assert not ax._calls
