"""axon_attn_shared at the ends of its range and by the library's own limit (nothing set in the environment)."""
import numpy as np
import pytest

import kv_model as km
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
