"""Own blocks that are rewritten between calls of axon_attn_shared: its second kernel starts before the one in front has
ended, and has to read what the copy before that wrote."""
import pytest

from test_gpu_shared import DEV, Case, ax, small_cases_share_too  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("H,G,d,dtype,rows", [(32, 8, 128, "bf16", 12), (14, 2, 64, "fp16", 40), (16, 1, 128, "bf16", 3)])
def test_what_a_copy_wrote_is_read(ax, H, G, d, dtype, rows, captured):  # noqa: F811
    """Each step fills a whole own block and the last, partly filled one of every row anew, then attends: the bits of the same
    step with the GPU waited for in between."""
    c = Case(H, G, d, dtype, [(800, [850 + i for i in range(rows)])], seed=rows, layers=1, layer=0)
    steps, spare = 40, 6
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    new = [torch.empty(1, spare * rows, G, 16, d, dtype=c.k.dtype, device=DEV).normal_(generator=g) for _ in range(2)]
    first = c.k.shape[1]
    k, v = (torch.cat([a, b], 1) for a, b in zip((c.k, c.v), new))
    cache = ax.make_kv_cache(k, v)
    work = ax.make_shared_workspace(cache, rows, H)
    own = torch.cat([c.bt[:, 51], torch.stack([c.bt[b, c.pos[b] // 16] for b in range(rows)])])
    r = torch.Generator().manual_seed(5)
    src = [first + torch.randperm(spare * rows, generator=r)[:2 * rows].to(DEV, torch.int32) for _ in range(steps)]
    outs, want = (torch.zeros(steps, rows, H, d, dtype=c.q.dtype, device=DEV) for _ in range(2))

    def step(i, out):
        ax.axon_kv_copy_blocks(cache, src[i], own)
        ax.axon_attn_shared(cache, 0, c.q, c.ctx, c.offsets, c.prefix, out, work, c.bt)

    for i in range(steps):
        ax.axon_kv_copy_blocks(cache, src[i], own)
        torch.cuda.synchronize()
        ax.axon_attn_shared(cache, 0, c.q, c.ctx, c.offsets, c.prefix, want[i], work, c.bt)
        torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    if captured:
        graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
            for i in range(steps):
                step(i, outs[i])
        torch.cuda.synchronize()
    for _ in range(10):
        outs.zero_()
        if captured:
            graph.replay()
        else:
            for i in range(steps):
                step(i, outs[i])
        assert torch.equal(outs, want)
