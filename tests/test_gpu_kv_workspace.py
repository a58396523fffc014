"""One workspace of the one-token attention over many calls: other shapes, batches, lengths and masks in turn, with rows
that are cut between workers and joined in one level and in two. Each call has to leave it fit for the next one."""
import pytest

from test_gpu_kv_attention import ULP, Case, close

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ax():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


def run(ax, c, work):
    out = torch.full_like(c.q, float("nan"))
    lse = torch.full((len(c.past), c.H), float("nan"), device="cuda")
    ax.axon_attn_decode(ax.make_kv_cache(c.k, c.v), c.layer, c.q, c.ctx, out, work, block_table=c.bt, window=c.window,
                        sinks=c.sinks, lse=lse, err=c.err)
    assert ax.axon_check_error(c.err) == (0, 0)
    return out, lse


def ticket_bytes():
    """The tickets stand in front, three per worker of the largest launch (three CTAs of four workers per SM)."""
    return 3 * 4 * 3 * 4 * torch.cuda.get_device_properties(0).multi_processor_count


def rows(past, *shape, **kw):
    return Case(*shape, past, [1] * len(past), kw.get("window", 0), kw.get("sinks", 0), seed=sum(past) % 1000 + shape[0])


CALLS = [
    lambda: rows([4095 + 4096 * b for b in range(8)], 4, 1, 128, "bf16"),       # joined in two levels, wide states
    lambda: rows([3000, 2900], 14, 2, 64, "fp16"),                              # narrow states, joined in one
    lambda: rows([9000], 16, 1, 64, "bf16"),                                    # 16 heads per kv head
    lambda: rows([700, 40, 0, 5000, 63] * 9, 8, 4, 64, "bf16", window=600, sinks=20),
    lambda: rows([20000, 7], 8, 1, 64, "fp16"),                                 # two levels, narrow states
    lambda: rows([1500 + b for b in range(64)], 32, 8, 128, "fp16", window=1000, sinks=4),
]


def test_a_workspace_serves_shapes_in_turn(ax):
    cases = [make() for make in CALLS]
    size = 0
    for c in cases:
        size = max(size, ax.make_attn_workspace(ax.make_kv_cache(c.k, c.v), len(c.past), c.H).numel())
    fresh = [run(ax, c, torch.zeros(size, dtype=torch.uint8, device="cuda")) for c in cases]
    for c, (o, _) in zip(cases[1:4], fresh[1:4]):
        close(o, c.reference()[0], c.vmax(), ULP[c.dtype])
    work = torch.zeros(size, dtype=torch.uint8, device="cuda")
    n = len(cases)
    for i in [0, 1, 0, 2, 1, 4, 3, 5, 0, 3, 1, 2, 5, 4, 1] + list(range(n)) + list(reversed(range(n))):
        o, lse = run(ax, cases[i], work)
        assert torch.equal(o, fresh[i][0]) and torch.equal(lse, fresh[i][1]), f"call of case {i}"
        assert not work[:ticket_bytes()].any(), f"tickets after case {i}"


def test_the_same_every_time_on_one_workspace(ax):
    """Batches, lengths and windows that change from call to call."""
    cases = [rows(p, 8, 2, 64, "bf16", window=w, sinks=s) for p, w, s in
             [([5000, 700, 64], 0, 0), ([16000], 0, 0), ([5000, 700, 64], 900, 4), ([30, 2, 1, 900] * 8, 0, 0), ([400], 128, 1)]]
    work = ax.make_attn_workspace(ax.make_kv_cache(cases[0].k, cases[0].v), 32, 8)
    first = [run(ax, c, work) for c in cases]
    for _ in range(3):
        for c, (o, lse) in zip(cases, first):
            a, la = run(ax, c, work)
            assert torch.equal(a, o) and torch.equal(la, lse)
            assert not work[:ticket_bytes()].any()


def test_the_size_does_not_depend_on_the_rows(ax):
    """Tickets go by workers: a workspace for one row serves any number."""
    c = rows([700 + b for b in range(40)], 8, 2, 64, "bf16")
    cache = ax.make_kv_cache(c.k, c.v)
    work = ax.make_attn_workspace(cache, 1, 8)
    assert work.numel() == ax.make_attn_workspace(cache, 2048, 8).numel()
    close(run(ax, c, work)[0], c.reference()[0], c.vmax(), ULP["bf16"])
