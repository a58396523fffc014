"""Infinities and NaN among the visible values of shared blocks: their dim of the output is not finite in any row that sees
them, however little the key weighs, as with axon_attn_decode; the other dims are right."""
import numpy as np
import pytest

from test_gpu_shared import DEV, TYPES, ULP, Case, ax, run, small_cases_share_too  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BAD = [(80, 3, 0, 5, float("nan")), (100, 15, 1, 9, float("inf")), (200, 0, 0, 11, float("-inf")), (127, 7, 1, 60, float("nan"))]


@pytest.mark.parametrize("rows", [3, 40])  # one tile and two
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_that_are_not_finite_show(ax, dtype, rows):  # noqa: F811
    """Blocks 64 to 127 of 256 weigh next to nothing: dim 0 of the queries is 8 and of these keys -256, so that their scores are
    181 - 30 below the others, 2^-217. Parts of the prefix pass of these alone have a factor of 0 in fp32.

    Scores of the other keys stay below 30 (dim 0 adds 8 * 4.5 / 128^0.5 = 3.2 at most), so the tolerance is test_gpu_shared's."""
    c = Case(8, 2, 128, dtype, [(4096, [4097 + 5 * i for i in range(rows)])], seed=31, layers=1, layer=0)
    c.q[:, :, 0] = 8.0
    blocks = c.bt[0, :256].long()
    c.k[0][blocks[64:128], :, :, 0] = -256.0
    clean = c.v.clone()
    hidden = {0: [], 1: []}
    for block, slot, head, dim, value in BAD:
        clean[0, blocks[block], head, slot, dim] = 0.0
        c.v[0, blocks[block], head, slot, dim] = value
        hidden[head].append(dim)
    held = c.k[0][c.bt.long().clamp(min=0)].transpose(2, 3).flatten(1, 2).double().cpu().numpy()
    seen = clean[0][c.bt.long().clamp(min=0)].transpose(2, 3).flatten(1, 2).double().cpu().numpy()
    c.keys, c.values = ([x[b, :p + 1] for b, p in enumerate(c.pos)] for x in (held, seen))
    some = sorted({0, 1, rows // 2, rows - 1})
    want, wlse = c.reference(some)
    cache = ax.make_kv_cache(c.k, c.v)
    work = ax.make_shared_workspace(cache, rows, 8)
    n = 144 * torch.cuda.get_device_properties(0).multi_processor_count + 16
    work[n:] = 255  # behind the counters anything may stand: parts that nobody writes are not read
    plain, lse = torch.empty_like(c.q), torch.empty(rows, 8, device=DEV)
    ax.axon_attn_decode(cache, 0, c.q, c.ctx, plain, ax.make_attn_workspace(cache, rows, 8), block_table=c.bt, lse=lse)
    vmax = max(np.abs(v).max() for v in c.values)
    for got, gl in ((plain, lse), run(ax, c, work=work)):
        got, gl = got.double().cpu().numpy(), gl.double().cpu().numpy()
        for h in range(8):
            dims = hidden[h // 4]
            rest = [x for x in range(128) if x not in dims]
            assert not np.isfinite(got[:, h, dims]).any()
            assert np.isfinite(got[:, h, rest]).all()
            off = np.abs(got[some][:, h, rest] - want[some][:, h, rest]) - ULP[dtype] * np.abs(want[some][:, h, rest])
            assert off.max() <= 5e-4 * vmax
        assert np.abs(gl[some] - wlse[some]).max() <= 5e-4
    assert ax.axon_check_error(c.err) == (0, 0)
