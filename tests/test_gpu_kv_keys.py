"""Which keys the attention on a paged cache counts, one by one: with queries of zero every visible key has the same
probability, and with values that are one in a single dim (the position's remainder) a dim of the output times the
number of visible keys is how many of them fall on it. A key too few or too many changes a count by one, however many
keys there are; rounding an output of at most 120 counts moves it by less than 120 * 2^-9 < 1 / 2."""
import numpy as np
import pytest

from test_gpu_kv_attention import Case

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


def counted(c):
    """Values as above in the case's cache; the counts of each query, [rows, d], and how many keys it sees."""
    d = c.d
    for b, total in enumerate(p + n for p, n in zip(c.past, c.new)):
        for j in range(-(-total // 16)):
            if c.table[b, j] < 0:
                continue
            n = min(16, total - 16 * j)
            ones = torch.nn.functional.one_hot((torch.arange(16 * j, 16 * j + n)) % d, d).to(c.v.dtype).cuda()
            c.v[c.layer, int(c.table[b, j]), :, :n] = ones
    c.q.zero_()
    want, seen = [], []
    for b, n in enumerate(c.new):
        for pos in range(c.past[b], c.past[b] + n):
            t = np.arange(pos + 1)
            if c.window:
                t = t[(t > pos - c.window) | (t < c.sinks)]
            want.append(np.bincount(t % d, minlength=d))
            seen.append(len(t))
    return np.array(want), np.array(seen)


def check(out, want, seen):
    got = out.double().cpu().numpy() * seen[:, None, None]
    assert want.max() <= 120
    assert np.array_equal(np.rint(got), np.broadcast_to(want[:, None, :], got.shape))


CASES = [([0], [700], 0, 0), ([2500, 37, 900], [9, 130, 1], 0, 0), ([4001], [33], 0, 0), ([1200], [260], 500, 20),
         ([3000, 640, 5], [17, 64, 200], 1111, 37), ([6100], [3], 0, 0), ([6000], [2], 5003, 4)]


@pytest.mark.parametrize("past,new,window,sinks", CASES)
@pytest.mark.parametrize("H,G,d,dtype", [(8, 2, 64, "bf16"), (9, 3, 64, "fp16"), (8, 1, 128, "bf16"), (5, 5, 128, "fp16")])
def test_chunks_count_every_key_once(ax, H, G, d, dtype, past, new, window, sinks):
    c = Case(H, G, d, dtype, past, new, window, sinks, seed=sum(past))
    want, seen = counted(c)
    out = torch.full_like(c.q, float("nan"))
    ax.axon_attn_prefill(ax.make_kv_cache(c.k, c.v), c.layer, c.q, c.cu, c.ctx, max(new), out, block_table=c.bt, window=window,
                         sinks=sinks, err=c.err)
    assert ax.axon_check_error(c.err) == (0, 0)
    check(out, want, seen)


@pytest.mark.parametrize("past,window,sinks", [([6100, 5, 640], 0, 0), ([7000], 5003, 4), ([900 + 7 * b for b in range(40)], 500, 20)])
@pytest.mark.parametrize("H,G,d,dtype", [(8, 2, 64, "bf16"), (16, 1, 128, "fp16")])
def test_single_tokens_count_every_key_once(ax, H, G, d, dtype, past, window, sinks):
    c = Case(H, G, d, dtype, past, [1] * len(past), window, sinks, seed=sum(past) % 999)
    want, seen = counted(c)
    cache = ax.make_kv_cache(c.k, c.v)
    out = torch.full_like(c.q, float("nan"))
    ax.axon_attn_decode(cache, c.layer, c.q, c.ctx, out, ax.make_attn_workspace(cache, len(past), H), block_table=c.bt,
                        window=window, sinks=sinks, err=c.err)
    assert ax.axon_check_error(c.err) == (0, 0)
    check(out, want, seen)


@pytest.mark.parametrize("entry", [-1, 10 ** 6])
def test_a_missing_block_spoils_its_own_rows_only(ax, entry):
    """A visible table entry that names no block is reported by both operators; rows that would have read it hold numbers of
    no meaning, finite ones, and the other rows what they should."""
    c = Case(8, 2, 64, "fp16", [100, 300, 40], [1, 1, 1], 0, 0, seed=3)
    want, seen = counted(c)
    c.bt[1, 4] = entry
    cache = ax.make_kv_cache(c.k, c.v)
    for op in ("decode", "prefill"):
        out = torch.full_like(c.q, float("nan"))
        if op == "decode":
            ax.axon_attn_decode(cache, c.layer, c.q, c.ctx, out, ax.make_attn_workspace(cache, 3, 8), block_table=c.bt, err=c.err)
        else:
            ax.axon_attn_prefill(cache, c.layer, c.q, c.cu, c.ctx, 1, out, block_table=c.bt, err=c.err)
        assert ax.axon_check_error(c.err) == (ax.AXON_ERR_DEVICE_CHECK, 2)
        assert torch.isfinite(out).all()
        check(out[[0, 2]], want[[0, 2]], seen[[0, 2]])
