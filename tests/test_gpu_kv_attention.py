"""Attention on a paged key/value cache (axon_attn_decode, axon_attn_prefill) against
attention in 64 bits, one query at a time (kv_model.attention).

Every slot of the pools that no query of a case may see holds NaN, and every table entry
that the mask hides is -1, so that a read of either shows.

Tolerances. Inputs are exact. Scores are fp32 sums of 128 products at most, of magnitude
sum |q k| * scale < 30: off by < 128 * 2^-24 * 30 = 2.3e-4, twice that on a probability's
ratio, which moves an output by at most that times max |v|: 5e-4 max |v|. The output's
rounding adds half a unit: 2^-9 (bf16) or 2^-12 + tail (fp16: 2^-11) of |o|, doubled here. The decode
form's probabilities have two 16-bit terms (2^-16 and less: inside the first bound); the chunk form's have
one, in numerator and denominator alike: 2 * 2^-9 (bf16), 2 * 2^-12 (fp16, taken as 2^-11) of
max |v| at most."""
import numpy as np
import pytest

import kv_model as km

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ULP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -10}
PROB = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def ax():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


class Case:
    """A cache with B rows of `past` + `new` tokens in shuffled blocks; only the blocks that a query sees exist."""

    def __init__(self, H, G, d, dtype, past, new, window, sinks, seed=0, layers=2, layer=1, per=None, paged=True, spare=3):
        r = np.random.default_rng(seed)
        self.H, self.G, self.d, self.window, self.sinks, self.layer = H, G, d, window, sinks, layer
        self.past, self.new, self.dtype = past, new, dtype
        total = [max(0, p + n) for p, n in zip(past, new)]
        self.per = per or max(1, max(-(-t // 16) for t in total))
        B = len(past)
        N = B * self.per + (spare if paged else 0)
        t16 = TYPES[dtype]
        k = torch.full((layers, N, G, 16, d), float("nan"), dtype=t16)
        v = k.clone()
        self.table = np.full((B, self.per), -1, dtype=np.int32)
        perm = r.permutation(N) if paged else np.arange(N)
        self.keys, self.values = [], []
        for b in range(B):
            kk = torch.from_numpy(r.standard_normal((total[b], G, d))).to(t16)
            vv = torch.from_numpy(r.standard_normal((total[b], G, d))).to(t16)
            self.keys.append(kk.double().numpy())
            self.values.append(vv.double().numpy())
            first = max(0, past[b] - window + 1) if window else 0  # of the first query
            for j in range(-(-total[b] // 16)):
                lo, hi = j * 16, min(total[b], j * 16 + 16)
                if paged and hi <= first and lo >= sinks:
                    continue  # hidden from every query: stays -1
                blk = perm[b * self.per + j]
                self.table[b, j] = blk
                k[layer, blk, :, :hi - lo] = kk[lo:hi].transpose(0, 1)
                v[layer, blk, :, :hi - lo] = vv[lo:hi].transpose(0, 1)
        self.k, self.v = k.cuda(), v.cuda()
        rows = sum(new)
        self.q = torch.from_numpy(r.standard_normal((rows, H, d)) * 1.6).to(t16).cuda()
        self.bt = torch.from_numpy(self.table).cuda() if paged else None
        self.ctx = torch.tensor(past, dtype=torch.int32, device="cuda")
        self.cu = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def reference(self, scale=None):
        q = self.q.double().cpu().numpy()
        o, lse, row = np.zeros(q.shape), np.full(q.shape[:2], -np.inf), 0
        for b, n in enumerate(self.new):
            for i in range(n):
                o[row], lse[row] = km.attention(q[row], self.keys[b], self.values[b], self.past[b] + i, self.window,
                                                self.sinks, scale)
                row += 1
        return o, lse

    def vmax(self):
        return max([np.abs(v).max() for v in self.values if v.size], default=0.0)


def close(got, want, vmax, ulp, prob=0.0):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    off = np.abs(got - want) - ulp * np.abs(want)
    bound = (5e-4 + prob) * vmax
    assert off.max(initial=0.0) <= bound, f"off by {off.max():.3e}, {bound:.3e} allowed"


def run_decode(ax, c, q=None, out=None, **kw):
    cache = ax.make_kv_cache(c.k, c.v)
    work = ax.make_attn_workspace(cache, len(c.past), c.H)
    q = c.q if q is None else q
    out = torch.full_like(c.q, float("nan")) if out is None else out
    lse = torch.full((len(c.past), c.H), float("nan"), device="cuda")
    per = dict(block_table=c.bt) if c.bt is not None else dict(blocks_per_seq=c.per)
    ax.axon_attn_decode(cache, c.layer, q, c.ctx, out, work, window=c.window, sinks=c.sinks, lse=lse, err=c.err, **per, **kw)
    tickets = work[-4 * len(c.past) * c.G:]
    torch.cuda.synchronize()
    assert not tickets.any(), "tickets are zero between calls"
    return out, lse


def check_decode(ax, c, **kw):
    out, lse = run_decode(ax, c, **kw)
    want, wlse = c.reference(kw.get("scale"))
    close(out, want, c.vmax(), ULP[c.dtype])
    lse = lse.double().cpu().numpy()
    empty = np.isinf(wlse)
    assert np.array_equal(np.isneginf(lse), empty)
    assert np.abs(lse[~empty] - wlse[~empty]).max(initial=0.0) <= 5e-4
    assert ax.axon_check_error(c.err) == (0, 0)


HEADS = [(14, 2, 64), (32, 8, 128), (9, 3, 64), (4, 4, 128), (10, 1, 128), (16, 1, 64), (5, 5, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,d", HEADS)
def test_decode_ragged_lengths(ax, H, G, d, dtype):
    past = [0, 1, 14, 15, 16, 17, 130, 577, 63, 64, 255]
    check_decode(ax, Case(H, G, d, dtype, past, [1] * len(past), 0, 0, seed=H * d))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (24, 16), (40, 33), (100, 5), (64, 64), (5, 1000),
                                          (4096, 4)])
@pytest.mark.parametrize("H,G,d", [(6, 2, 128), (12, 1, 64)])
def test_decode_window_and_sinks(ax, H, G, d, window, sinks):
    past = [0, 3, 15, 16, 39, 40, 41, 63, 64, 100, 117, 300, 601]
    check_decode(ax, Case(H, G, d, "bf16", past, [1] * len(past), window, sinks, seed=window))


def test_sinks_without_a_window_change_nothing(ax):
    c = Case(8, 2, 64, "fp16", [100, 31], [1, 1], 0, 7, seed=3)
    check_decode(ax, c)


@pytest.mark.parametrize("past", [[-1, 40, -5, 0], [-1], [-1, -1, -1]])
def test_decode_idle_rows(ax, past):
    c = Case(8, 2, 128, "bf16", past, [1] * len(past), 0, 0, seed=8, per=4)
    check_decode(ax, c)


@pytest.mark.parametrize("B,past", [(1, 9000), (2, 3000), (3, 4095)])
@pytest.mark.parametrize("H,G,d", [(8, 1, 64), (16, 2, 128)])
def test_decode_long_rows_are_split_and_joined(ax, B, past, H, G, d):
    check_decode(ax, Case(H, G, d, "fp16", [past - 7 * b for b in range(B)], [1] * B, 0, 0, seed=B))


def test_decode_one_long_row_among_many_short(ax):
    past = [20000] + [5 + 3 * b for b in range(150)]
    check_decode(ax, Case(4, 2, 64, "bf16", past, [1] * len(past), 0, 0, seed=4))


def test_decode_many_rows(ax):
    past = [(7 * b) % 90 for b in range(700)]
    check_decode(ax, Case(3, 1, 64, "fp16", past, [1] * len(past), 50, 3, seed=5))


def test_decode_contiguous_rows(ax):
    check_decode(ax, Case(8, 4, 64, "bf16", [100, 5, 64], [1] * 3, 0, 0, seed=6, paged=False))


@pytest.mark.parametrize("scale", [0.03, 0.5])
def test_decode_scale(ax, scale):
    c = Case(8, 4, 64, "fp16", [100, 5], [1] * 2, 0, 0, seed=6)
    c.q.mul_(0.25)
    check_decode(ax, c, scale=scale)


def test_decode_is_the_same_every_time(ax):
    c = Case(16, 2, 128, "bf16", [5000, 700, 64], [1] * 3, 0, 0, seed=9)
    a, la = run_decode(ax, c)
    for _ in range(3):
        b, lb = run_decode(ax, c)
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_decode_strides_and_another_stream(ax):
    """Queries inside a fused [q | k | v] row with heads apart, outputs inside a wider buffer, on a stream of their own."""
    c = Case(8, 2, 64, "bf16", [100, 30, 77], [1] * 3, 0, 0, seed=7)
    wide = torch.full((3, 12, 72), float("nan"), dtype=c.q.dtype, device="cuda")
    wide[:, 2:10, :64] = c.q
    out = torch.full((3, 10, 80), 7.0, dtype=c.q.dtype, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o, _ = run_decode(ax, c, q=wide[:, 2:10, :64], out=out[:, 1:9, :64], stream=s)
    close(o, c.reference()[0], c.vmax(), ULP["bf16"])
    out[:, 1:9, :64] = 7.0
    assert (out == 7.0).all()


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 2 ** 31 - 1), (20, 2 ** 31 - 1), (2 ** 31 - 1, 3)])
def test_largest_windows_and_sinks(ax, window, sinks):
    c = Case(4, 2, 64, "bf16", [100, 30], [1, 1], 0, 0, seed=7)
    c.window, c.sinks = window, sinks
    check_decode(ax, c)
    check_prefill(ax, c)


def test_heads_before_rows(ax):
    """Queries and outputs stored [heads, rows, head_dim], and every second row of a buffer."""
    c = Case(8, 2, 64, "fp16", [40, 9, 0], [1, 1, 1], 0, 0, seed=17)
    want = c.reference()[0]
    q = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.full((8, 3, 64), float("nan"), dtype=c.q.dtype, device="cuda").transpose(0, 1)
    assert q.stride() == (64, 192, 1)
    close(run_decode(ax, c, q=q, out=out)[0], want, c.vmax(), ULP["fp16"])
    out.fill_(float("nan"))
    check_prefill(ax, c, q=q, out=out)
    wide = torch.full((6, 8, 64), float("nan"), dtype=c.q.dtype, device="cuda")
    wide[::2] = c.q
    check_prefill(ax, c, q=wide[::2], out=torch.empty_like(wide)[::2])
    close(run_decode(ax, c, q=wide[::2], out=torch.empty_like(wide)[::2])[0], want, c.vmax(), ULP["fp16"])


def test_decode_shows_an_infinite_value(ax):
    """An infinite value at a visible token: its dim of the output is not finite, the others are untouched."""
    c = Case(4, 1, 64, "bf16", [40], [1], 0, 0, seed=11)
    blk = int(c.table[0, 1])
    c.v[1, blk, 0, 3, 5] = float("inf")
    out, _ = run_decode(ax, c)
    assert not torch.isfinite(out[0, :, 5]).any()
    assert torch.isfinite(out[0, :, :5]).all() and torch.isfinite(out[0, :, 6:]).all()


@pytest.mark.parametrize("entry", [-1, 10 ** 6, -2 ** 31])
def test_decode_reports_block_numbers_out_of_range(ax, entry):
    c = Case(4, 1, 64, "bf16", [40, 20], [1, 1], 0, 0, seed=12)
    c.bt[0, 1] = entry
    out, _ = run_decode(ax, c)
    assert ax.axon_check_error(c.err) == (ax.AXON_ERR_DEVICE_CHECK, 2)
    assert ax.axon_check_error(c.err) == (0, 0)
    want, _ = c.reference()
    close(out[1:], want[1:], c.vmax(), ULP["bf16"])


@pytest.mark.parametrize("pos", [64, 2 ** 31 - 1])
def test_decode_reports_positions_past_the_table(ax, pos):
    c = Case(4, 1, 64, "bf16", [63, 20], [1, 1], 0, 0, seed=13)
    c.ctx[0] = pos
    out, lse = run_decode(ax, c)
    assert ax.axon_check_error(c.err) == (ax.AXON_ERR_DEVICE_CHECK, 4)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()
    close(out[1:], c.reference()[0][1:], c.vmax(), ULP["bf16"])


# ---------------------------------------------------------------- chunks


def check_prefill(ax, c, q=None, out=None, stream=None):
    cache = ax.make_kv_cache(c.k, c.v)
    q = c.q if q is None else q
    out = torch.full_like(c.q, float("nan")) if out is None else out
    per = dict(block_table=c.bt) if c.bt is not None else dict(blocks_per_seq=c.per)
    ax.axon_attn_prefill(cache, c.layer, q, c.cu, c.ctx, max(c.new), out, window=c.window, sinks=c.sinks, err=c.err,
                         stream=stream, **per)
    torch.cuda.synchronize()
    close(out, c.reference()[0], c.vmax(), ULP[c.dtype], PROB[c.dtype])
    assert ax.axon_check_error(c.err) == (0, 0)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,d", HEADS)
def test_prefill_ragged_chunks(ax, H, G, d, dtype):
    check_prefill(ax, Case(H, G, d, dtype, [0, 5, 100, 0, 33, 16], [1, 40, 7, 150, 16, 0], 0, 0, seed=H + d))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 2), (16, 4), (24, 16), (40, 33), (100, 5), (64, 64), (5, 1000), (130, 4)])
@pytest.mark.parametrize("H,G,d", [(6, 2, 128), (9, 3, 64)])
def test_prefill_window_and_sinks(ax, H, G, d, window, sinks):
    check_prefill(ax, Case(H, G, d, "fp16", [0, 300, 77, 40], [290, 33, 1, 16], window, sinks, seed=window))


def test_prefill_long_context_behind_a_short_chunk(ax):
    check_prefill(ax, Case(8, 1, 128, "bf16", [2000, 1500], [5, 30], 0, 0, seed=2))
    check_prefill(ax, Case(8, 1, 128, "bf16", [2000, 1500], [5, 30], 600, 20, seed=2))


@pytest.mark.parametrize("past,new", [([1030], [3]), ([1300, 900], [17, 40]), ([2040, 5, 1100], [9, 30, 1]), ([4000], [100]),
                                      ([3000, 1279], [1, 1])])
@pytest.mark.parametrize("H,G,d,window,sinks", [(8, 2, 128, 0, 0), (9, 3, 64, 0, 0), (14, 2, 64, 1500, 20), (5, 5, 128, 2500, 3)])
def test_prefill_few_rows_behind_long_contexts(ax, past, new, H, G, d, window, sinks):
    """Items that a cluster of 2, 4 or 8 CTAs shares, beside ones that are too short for it."""
    check_prefill(ax, Case(H, G, d, "fp16", past, new, window, sinks, seed=sum(past)))


def test_prefill_short_rows_in_a_wide_table(ax):
    check_prefill(ax, Case(8, 2, 64, "bf16", [0, 60, 1200], [20, 1, 5], 0, 0, seed=3, per=400))


def test_prefill_is_the_same_every_time(ax):
    c = Case(8, 2, 128, "bf16", [2500, 1100], [30, 9], 0, 0, seed=9)
    a = check_prefill(ax, c)
    for _ in range(3):
        assert torch.equal(a, check_prefill(ax, c))


def test_prefill_shows_a_score_far_above_the_first_ones(ax):
    """The bound of a row's scores comes from its first step: later keys that exceed it by hundreds have to raise it."""
    for past, new in (([0], [700]), ([1800], [4])):
        c = Case(4, 2, 128, "fp16", past, new, 0, 0, seed=5)
        for b, t in ((0, 200), (0, 201), (0, past[0] + new[0] - 2)):
            blk = int(c.table[b, t // 16])
            c.k[1, blk, :, t % 16] *= 40.0
            c.keys[b][t] = c.k[1, blk, :, t % 16].double().cpu().numpy()
        out = torch.full_like(c.q, float("nan"))
        cache = ax.make_kv_cache(c.k, c.v)
        ax.axon_attn_prefill(cache, 1, c.q, c.cu, c.ctx, max(c.new), out, block_table=c.bt, err=c.err)
        # scores of up to 40 * 30: off by 40 times as much, where neighbours are that close
        close(out, c.reference()[0], 40 * c.vmax(), ULP["fp16"], PROB["fp16"] / 40)
        assert ax.axon_check_error(c.err) == (0, 0)


def test_prefill_contiguous_rows(ax):
    check_prefill(ax, Case(4, 2, 64, "bf16", [10, 0], [30, 64], 20, 1, seed=6, paged=False))


def test_prefill_strides_and_another_stream(ax):
    c = Case(8, 2, 64, "bf16", [10, 0], [30, 21], 0, 0, seed=7)
    wide = torch.full((51, 12, 72), float("nan"), dtype=c.q.dtype, device="cuda")
    wide[:, 2:10, :64] = c.q
    out = torch.full((51, 10, 80), 7.0, dtype=c.q.dtype, device="cuda")
    torch.cuda.synchronize()
    check_prefill(ax, c, q=wide[:, 2:10, :64], out=out[:, 1:9, :64], stream=torch.cuda.Stream())
    out[:, 1:9, :64] = 7.0
    assert (out == 7.0).all()


def test_a_chunk_of_one_is_a_decode_row(ax):
    c = Case(8, 2, 128, "fp16", [100, 31, 0, 640], [1] * 4, 200, 4, seed=21)
    a, _ = run_decode(ax, c)
    b = check_prefill(ax, c)
    assert (a.double() - b.double()).abs().max() <= (PROB["fp16"] + ULP["fp16"]) * c.vmax()


@pytest.mark.parametrize("cu,ctx,bit", [([0, 5, 21], [0, 8], 16), ([1, 10, 20], [0, 8], 16), ([0, 12, 8], [0, 8], 16),
                                        ([0, 10, 20], [-3, 8], 4), ([0, 10, 20], [0, 2 ** 31 - 4], 4),
                                        ([0, 10, 20], [0, 60], 4)])
def test_prefill_reports_inconsistent_offsets_and_positions(ax, cu, ctx, bit):
    c = Case(4, 1, 64, "bf16", [0, 8], [10, 10], 0, 0, seed=14, per=4)
    c.cu.copy_(torch.tensor(cu, dtype=torch.int32))
    c.ctx.copy_(torch.tensor(ctx, dtype=torch.int32))
    cache = ax.make_kv_cache(c.k, c.v)
    out = torch.zeros_like(c.q)
    ax.axon_attn_prefill(cache, c.layer, c.q, c.cu, c.ctx, 15, out, block_table=c.bt, err=c.err)
    assert ax.axon_check_error(c.err) == (ax.AXON_ERR_DEVICE_CHECK, bit)


def test_prefill_reports_block_numbers_out_of_range(ax):
    c = Case(4, 1, 64, "bf16", [0, 40], [10, 10], 0, 0, seed=15)
    c.bt[1, 1] = 10 ** 6
    cache = ax.make_kv_cache(c.k, c.v)
    out = torch.zeros_like(c.q)
    ax.axon_attn_prefill(cache, c.layer, c.q, c.cu, c.ctx, 10, out, block_table=c.bt, err=c.err)
    assert ax.axon_check_error(c.err) == (ax.AXON_ERR_DEVICE_CHECK, 2)
    close(out[:10], c.reference()[0][:10], c.vmax(), ULP["bf16"], PROB["bf16"])


def test_offsets_past_32_bits(ax):
    """Blocks at the end of a pool of more than 2^31 elements, in the second of two layers."""
    H, G, d, N = 16, 8, 128, 70000
    c = Case(H, G, d, "bf16", [37, 18], [1, 1], 0, 0, seed=30)
    k = torch.empty(2, N, G, 16, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    n = c.k.shape[1]
    k[1, N - n:], v[1, N - n:] = c.k[1], c.v[1]
    c.k, c.v, c.bt = k, v, torch.where(c.bt >= 0, c.bt + (N - n), c.bt)
    check_decode(ax, c)
    check_prefill(ax, c)


def test_the_binding_refuses(ax):
    c = Case(4, 2, 64, "bf16", [10, 5], [1, 1], 0, 0, seed=1)
    cache = ax.make_kv_cache(c.k, c.v)
    work = ax.make_attn_workspace(cache, 2, 4)
    ok = dict(block_table=c.bt)
    out = torch.empty_like(c.q)
    for bad in (dict(q=c.q.half()), dict(q=c.q.cpu()), dict(out=out[:1]), dict(out=out.float()), dict(ctx=c.ctx.long()),
                dict(ctx=c.ctx[:1]), dict(q=c.q.transpose(1, 2)), dict(lse=torch.empty(2, 4, dtype=torch.float64, device="cuda"))):
        a = dict(q=c.q, ctx=c.ctx, out=out, lse=None)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            ax.axon_attn_decode(cache, 0, a["q"], a["ctx"], a["out"], work, lse=a["lse"], **ok)
    with pytest.raises(TypeError):
        ax.axon_attn_decode(cache, 0, c.q, c.ctx, out, work, block_table=c.bt.t())
    with pytest.raises(ax.AxonError):
        ax.axon_attn_decode(cache, 0, c.q, c.ctx, out, work[:-16], **ok)
    with pytest.raises(ax.AxonError):
        ax.axon_attn_decode(cache, 2, c.q, c.ctx, out, work, **ok)
