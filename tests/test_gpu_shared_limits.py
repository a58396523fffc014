"""axon_attn_shared at the ends of its range and by the library's own limit (nothing set in the environment)."""
import numpy as np
import pytest

import kv_model as km
import test_gpu_shared as sh
from test_gpu_shared import DEV, ax  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def the_own_limit(monkeypatch):
    monkeypatch.delenv("AXON_SHARED_MIN_BYTES", raising=False)


def test_millions_of_own_pages(ax):  # noqa: F811
    """4.2 million pages of own parts, more than fp32 counts with the weight that the division of the SMs gives them: all CTAs cut
    them alike, and the counters are zero again. The rows' tables name the same few blocks, in another order each.

    Against the one-token form, whose tolerance is this form's too: scores below 30 and off by 2.3e-4, 5e-4 max |v| per side, and
    half a unit of bf16 each; two rows against 64 bits, with one side's."""
    B, H, G, d, whole, own = 128, 16, 8, 128, 256, 4096
    r = np.random.default_rng(71)
    g = torch.Generator(device=DEV)
    g.manual_seed(71)
    N = whole + own + B
    k, v = (torch.empty(1, N, G, 16, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    q = torch.empty(B, H, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) * 1.6
    table = np.concatenate([np.tile(np.arange(whole), (B, 1)), np.stack([whole + r.permutation(own + B)[:own] for _ in range(B)])], 1)
    bt = torch.from_numpy(table.astype(np.int32)).to(DEV)
    pos = (whole + own) * 16 - 1 - r.integers(0, 200, B)
    ctx = torch.from_numpy(pos.astype(np.int32)).to(DEV)
    assert B * G * own * 5 > 2 ** 24
    cache = ax.make_kv_cache(k, v)
    work = ax.make_shared_workspace(cache, B, H)
    a, again, b = (torch.empty_like(q) for _ in range(3))
    offsets, prefix = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, B], [whole * 16]))
    ax.axon_attn_shared(cache, 0, q, ctx, offsets, prefix, a, work, bt)
    ax.axon_attn_shared(cache, 0, q, ctx, offsets, prefix, again, work, bt)
    assert torch.equal(a, again)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert not work[:144 * sms + 16].any()  # tickets and counters
    ax.axon_attn_decode(cache, 0, q, ctx, b, work, block_table=bt)
    assert not torch.equal(a, b)  # other sums: the prefix pass ran
    vmax = float(v.abs().max())
    assert ((a.double() - b.double()).abs() <= 2 * 5e-4 * vmax + 2.0 ** -7 * b.double().abs()).all()
    for row in (0, 101):
        n = int(pos[row]) + 1
        keys, values = (x[0][bt[row].long()].transpose(1, 2).reshape(-1, G, d)[:n].double().cpu().numpy() for x in (k, v))
        want, _ = km.attention(q[row].double().cpu().numpy(), keys, values, n - 1)
        off = np.abs(a[row].double().cpu().numpy() - want) - 2.0 ** -8 * np.abs(want)
        assert off.max() <= 5e-4 * vmax


@pytest.mark.parametrize("text,shares", [("0", True), ("1000", True), ("99999999999999999999", False), ("", False), ("none", False),
                                         ("-1", False), ("0x0", False), ("10 MB", False), (" 0", False)])
def test_what_the_environment_may_say(ax, monkeypatch, text, shares):  # noqa: F811
    """A limit is a whole number; other text leaves the library's own, by which a case of this size shares nothing."""
    c = sh.Case(8, 2, 64, "bf16", [(300, [310, 320, 330]), (200, [250, 260])], seed=72)
    monkeypatch.setenv("AXON_SHARED_MIN_BYTES", text)
    out, _ = sh.run(ax, c)
    cache = ax.make_kv_cache(c.k, c.v)
    plain = torch.empty_like(c.q)
    ax.axon_attn_decode(cache, c.layer, c.q, c.ctx, plain, ax.make_attn_workspace(cache, 5, 8), block_table=c.bt)
    assert torch.equal(out, plain) != shares  # other sums where the prefix pass runs


@pytest.mark.parametrize("window,sinks", [(0, 0), (2300, 4)])
@pytest.mark.parametrize("rows,blocks,shares", [(16, 137, True), (16, 136, False), (65, 32, True), (64, 32, False), (17, 128, True)])
def test_about_the_limit(ax, rows, blocks, shares, window, sinks):  # noqa: F811
    """128 MB are 2048 reads of a block of 8 heads of 128 with keys and values; under a table that is wide enough for more the
    device finds out. Either way the rows are right, some of them against 64 bits."""
    c = sh.Case(32, 8, 128, "bf16", [(16 * blocks, [16 * blocks + 3 + 2 * (i % 9) for i in range(rows)])], window, sinks, seed=rows,
                layers=1, layer=0)
    assert (blocks * (rows - 1) >= 2048) == shares
    some = [0, rows // 2, rows - 1]
    cache = ax.make_kv_cache(c.k, c.v)
    plain = torch.empty_like(c.q)
    ax.axon_attn_decode(cache, 0, c.q, c.ctx, plain, ax.make_attn_workspace(cache, rows, 32), block_table=c.bt, window=window, sinks=sinks)
    for per in (c.per, 400):
        c.bt = torch.nn.functional.pad(c.bt, (0, per - c.bt.shape[1]), value=-1)
        sh.check(ax, c, rows=some)
        assert torch.equal(sh.run(ax, c)[0], plain) != shares


@pytest.mark.parametrize("rows", [2, 3])
def test_most_rows_and_groups_of_the_widest_heads(ax, monkeypatch, rows):  # noqa: F811
    """2048 rows in as many groups as they make, 16 query heads per kv head of 128 dims: the most shared memory that a call takes."""
    monkeypatch.setenv("AXON_SHARED_MIN_BYTES", "0")
    groups = [(160, [165 + i for i in range(rows)])] * (2048 // rows)
    c = sh.Case(16, 1, 128, "fp16", groups + [(0, [40])] * (2048 % rows), seed=73, layers=1, layer=0)
    assert len(c.pos) == 2048 and c.prefix.numel() <= 1024
    sh.check(ax, c, rows=[0, 1, 1000, 2046, 2047])
