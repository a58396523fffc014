"""New tokens into a paged cache (axon_kv_append) against rotation in 64 bits on the host, slot by slot.

Tolerance. A turned value is x c - y s with cosine and sine rounded to fp32 (2^-25 of at most 1, twice that allowed for
the angle) and two fp32 products and a sum: off by at most 4 * 2^-24 (|x| + |y|). Rounding to the cache's type adds
half a step of the result, eps / 2. What is not turned has the same bits. Slots that no token goes to hold what they
held, bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BITS = {"bf16": torch.int16, "fp16": torch.int16, "fp32": torch.int32}
DEV = "cuda"


@pytest.fixture(scope="module")
def ax():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


def frequencies(dim, theta=1e4, factor=0.0, low=1.0, high=4.0, original=64):
    f = theta ** (-np.arange(0, dim, 2) / dim)
    if factor:
        w = 2 * np.pi / f
        t = (original / w - low) / (high - low)
        f = np.where(w > original / low, f / factor, np.where(w < original / high, f, (1 - t) * f / factor + t * f))
    return f


def angles(positions, dim, **kw):
    return positions[:, None] * frequencies(dim, **kw)


def turned(x, pos, dim, interleaved, **kw):
    """x [rows, heads, d] in 64 bits with its first `dim` dims turned, and the bound's |x| + |y|."""
    a = angles(pos.astype(np.float64), dim, **kw)[:, None]
    out, size = x.copy(), np.zeros_like(x)
    i, j = (np.arange(0, dim, 2), np.arange(1, dim, 2)) if interleaved else (np.arange(dim // 2), np.arange(dim // 2, dim))
    out[..., i] = x[..., i] * np.cos(a) - x[..., j] * np.sin(a)
    out[..., j] = x[..., j] * np.cos(a) + x[..., i] * np.sin(a)
    size[..., i] = size[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return out, size


class Case:
    """`new` tokens of each row after `past` ones; the blocks are shuffled, pools hold a pattern."""

    def __init__(self, H, G, d, dtype, past, new, seed=0, layers=2, layer=1, per=None, paged=True):
        r = np.random.default_rng(seed)
        self.H, self.G, self.d, self.dtype, self.layer, self.past, self.new = H, G, d, dtype, layer, past, new
        self.t = TYPES[dtype]
        B = len(past)
        self.per = per or max(1, max(-(-(p + n) // 16) for p, n in zip(past, new)))
        N = B * self.per + (3 if paged else 0)
        self.k = torch.from_numpy(r.standard_normal((layers, N, G, 16, d))).to(self.t).to(DEV)
        self.v = torch.from_numpy(r.standard_normal((layers, N, G, 16, d))).to(self.t).to(DEV)
        self.table = (r.permutation(N)[:B * self.per] if paged else np.arange(N)).reshape(B, self.per).astype(np.int32)
        self.bt = torch.from_numpy(self.table).to(DEV) if paged else None
        T = sum(new)
        self.qkv = torch.from_numpy(r.standard_normal((T, H + 2 * G, d)) * 3).to(self.t).to(DEV)
        self.ctx = torch.tensor(past, dtype=torch.int32, device=DEV)
        self.cu = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def parts(self):
        H, G = self.H, self.G
        return self.qkv[:, :H], self.qkv[:, H:H + G], self.qkv[:, H + G:]

    def places(self):
        """(row of the packed batch, sequence, position) of every token."""
        out, row = [], 0
        for b, (p, n) in enumerate(zip(self.past, self.new)):
            out += [(row + i, b, p + i) for i in range(n)]
            row += n
        return out


def host(t):
    return t.detach().double().cpu().numpy()


def run(ax, c, rope, interleaved=False, chunks=True, out=None, queries=True, **kw):
    cache = ax.make_kv_cache(c.k, c.v)
    q, k, v = c.parts()
    out = torch.zeros(q.shape, dtype=c.t, device=DEV) if out is None else out
    per = dict(block_table=c.bt) if c.bt is not None else dict(blocks_per_seq=c.per)
    ax.axon_kv_append(cache, c.layer, k, v, c.ctx, cu_seqlens=c.cu if chunks else None, rope=rope, interleaved=interleaved,
                      q=q if queries else None, q_out=out if queries else None, err=c.err, **per, **kw)
    return out


def check(ax, c, dim, interleaved=False, chunks=True, skip=(), queries=True, out=None, freq={}, err=0, keys_skip=()):
    """skip: sequences that are left out; keys_skip: sequences whose keys and values are."""
    most = c.per * 16
    rope = ax.axon_rope_table(most, dim, freq.get("theta", 1e4), freq.get("factor", 0.0), original=freq.get("original", 64)) if dim else None
    k0, v0, x = c.k.clone(), c.v.clone(), c.qkv.clone()
    o = run(ax, c, rope, interleaved, chunks, out, queries)
    H, G = c.H, c.G
    places = [p for p in c.places() if p[1] not in skip]
    pos = np.zeros(x.shape[0], dtype=np.int64)
    for row, _, p in places:
        pos[row] = p
    want = host(x)
    size = np.zeros_like(want)
    if dim:
        want[:, :H + G], size[:, :H + G] = turned(want[:, :H + G], pos, dim, interleaved, **freq)
    off = 4 * 2.0 ** -24 * size + torch.finfo(c.t).eps / 2 * np.abs(want) * (size > 0) * (1 + 2.0 ** -20)
    got, rows = host(o), [row for row, _, _ in places]
    if queries:
        bound = off[rows, :H]
        assert (np.abs(got[rows] - want[rows, :H]) <= bound).all()
        left = sorted(set(range(x.shape[0])) - set(rows))
        assert not got[left].any()  # rows that are left out are not written
    k, v = host(c.k[c.layer]), host(c.v[c.layer])
    free = torch.ones(c.k.shape[1], 16, dtype=torch.bool)
    for row, b, p in places:
        if b in keys_skip:
            continue
        blk, i = c.table[b, p // 16], p % 16
        free[blk, i] = False
        assert (np.abs(k[blk, :, i] - want[row, H:H + G]) <= off[row, H:H + G]).all(), (row, b, p)
        assert (v[blk, :, i] == want[row, H + G:]).all(), (row, b, p)
    bits = BITS[c.dtype]
    for now, was in ((c.k, k0), (c.v, v0)):
        same = (now.view(bits) == was.view(bits)).all(-1).cpu()  # [layers, blocks, G, 16]
        assert same[[i for i in range(same.shape[0]) if i != c.layer]].all()
        assert same[c.layer].all(1)[free].all()
    assert ax.axon_check_error(c.err)[1] == err


HEADS = [(14, 2, 64), (32, 8, 128), (9, 3, 64), (5, 5, 128), (16, 1, 64)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("H,G,d", HEADS)
def test_one_token_per_row(ax, H, G, d, dtype):
    past = [0, 1, 14, 15, 16, 17, 130, 577, 63]
    check(ax, Case(H, G, d, dtype, past, [1] * len(past), seed=H), d, chunks=False)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dim", [(64, 16), (64, 64), (128, 32), (128, 64), (128, 112), (128, 128), (64, 0)])
def test_chunks_layouts_and_partial_rotation(ax, d, dim, interleaved, dtype):
    c = Case(6, 2, d, dtype, [0, 5, 100, 31, 16, 40], [33, 1, 0, 17, 16, 90], seed=dim)
    check(ax, c, dim, interleaved)


def test_scaled_frequencies(ax):
    check(ax, Case(6, 2, 128, "fp32", [0, 300, 4000], [33, 70, 90], seed=3), 128, freq=dict(theta=5e5, factor=8.0, original=512))


def test_table_of_far_positions(ax):
    for kw in (dict(theta=1e4), dict(theta=5e5, factor=8.0, original=8192)):
        t = host(ax.axon_rope_table(131072, 128, kw["theta"], kw.get("factor", 0.0), original=kw.get("original", 64)))
        a = angles(np.arange(131072.0), 128, **kw)
        assert np.abs(t[..., 0] - np.cos(a)).max() <= 2.0 ** -24
        assert np.abs(t[..., 1] - np.sin(a)).max() <= 2.0 ** -24


@pytest.mark.parametrize("H,G,d", [(32, 8, 128), (9, 3, 64)])
def test_long_chunks(ax, H, G, d):
    check(ax, Case(H, G, d, "bf16", [3, 7], [1501, 700], seed=5), d)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
def test_many_tokens_of_other_types(ax, dtype, interleaved):
    """Three heads per thread, 42 = 14 x 3 of them and 43 x 3 - 1; a part of the dims turned."""
    check(ax, Case(32, 5, 128, dtype, [3, 0, 40], [700, 1, 333], seed=8), 96, interleaved)
    check(ax, Case(100, 14, 64, dtype, [9], [600], seed=9), 64, interleaved)


def test_rows_in_place(ax):
    c = Case(8, 2, 64, "bf16", [3, 77], [20, 1], seed=6)
    q = c.parts()[0]
    want, _ = turned(host(q), np.array([3 + i for i in range(20)] + [77]), 64, False)
    rest = c.qkv[:, 8:].clone()
    run(ax, c, ax.axon_rope_table(c.per * 16, 64, 1e4), out=q)
    assert np.abs(host(q) - want).max() <= 2.0 ** -8 * np.abs(want).max()
    assert torch.equal(rest, c.qkv[:, 8:])


def test_keys_and_values_alone(ax):
    check(ax, Case(8, 2, 64, "fp16", [3, 77], [20, 1], seed=7), 64, queries=False)


def test_contiguous_rows_and_no_rotation(ax):
    check(ax, Case(4, 4, 128, "bf16", [0, 30, 15], [5, 1, 40], seed=8, paged=False), 0)
    check(ax, Case(4, 4, 128, "fp32", [0, 30, 15], [1, 1, 1], seed=8, paged=False), 64, chunks=False)


def test_bits_that_are_not_numbers_pass_through(ax):
    c = Case(4, 2, 64, "bf16", [0, 30], [17, 3], seed=9)
    bits = torch.randint(-32768, 32768, c.qkv.shape, dtype=torch.int16, device=DEV)
    c.qkv.copy_(bits.view(torch.bfloat16))
    bits = c.qkv.view(torch.int16).clone()
    out = run(ax, c, None)
    assert torch.equal(out.view(torch.int16), bits[:, :4])
    for row, b, p in c.places():
        blk = int(c.table[b, p // 16])
        assert torch.equal(c.k[c.layer, blk, :, p % 16].view(torch.int16), bits[row, 4:6])
        assert torch.equal(c.v[c.layer, blk, :, p % 16].view(torch.int16), bits[row, 6:])


def test_idle_rows_and_rows_past_the_table(ax):
    c = Case(8, 2, 64, "bf16", [5, 20, 40, 63, 2], [1] * 5, per=4)
    c.ctx.copy_(torch.tensor([5, -1, 40, 64, 2], dtype=torch.int32))
    check(ax, c, 64, chunks=False, skip=(1, 3), err=4)


def test_rows_past_the_rotary_table(ax):
    c = Case(8, 2, 64, "bf16", [5, 20, 40], [1] * 3, per=4)
    rope = ax.axon_rope_table(40, 64, 1e4)
    k0 = c.k.clone()
    out = run(ax, c, rope, chunks=False)
    assert out[:2].any() and not out[2].any()
    assert ax.axon_check_error(c.err)[1] == 4
    assert (c.k != k0).any(-1).sum() == 2 * c.G


def test_blocks_out_of_range(ax):
    c = Case(8, 2, 64, "bf16", [5, 20, 40, 50], [1, 1, 1, 1], per=4)
    c.bt[1, 1] = -1
    c.bt[2, 2] = c.k.shape[1]
    check(ax, c, 64, chunks=False, keys_skip=(1, 2), err=2)


def test_chunks_that_do_not_fit_are_left_out(ax):
    c = Case(8, 2, 64, "bf16", [5, 60, 0], [3, 5, 9], per=4)  # the second one's last token lies past the table
    check(ax, c, 64, skip=(1,), err=4)
    c = Case(8, 2, 64, "bf16", [5, 20, 0], [3, 5, 9], per=4)
    c.ctx[1] = -1
    check(ax, c, 64, skip=(1,), err=4)


def test_offsets_that_do_not_fit(ax):
    c = Case(8, 2, 64, "bf16", [5, 20, 0], [3, 5, 9], per=4)
    c.cu[3] = 14  # rows behind the last sequence
    rope = ax.axon_rope_table(64, 64, 1e4)
    out = run(ax, c, rope)
    assert out[:14].any(-1).all() and not out[14:].any() and ax.axon_check_error(c.err)[1] == 16
    c.cu.copy_(torch.tensor([0, 9, 3, 17], dtype=torch.int32))  # the second chunk ends before it begins
    out = run(ax, c, rope)
    assert ax.axon_check_error(c.err)[1] == 16
    c.cu.copy_(torch.tensor([-4, 3, 8, 1 << 30], dtype=torch.int32))
    out = run(ax, c, rope)
    assert not out[:3].any() and out[3:8].any(-1).all() and not out[8:].any()
    assert ax.axon_check_error(c.err)[1] == 16


def test_pools_past_two_to_the_31_elements(ax):
    G, d, N = 8, 128, 140000  # 2.29e9 elements
    k = torch.empty(1, N, G, 16, d, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    k[0, -1], v[0, -1] = 0, 0
    cache = ax.make_kv_cache(k, v)
    x = torch.randn(1, 3 * G, d, device=DEV).bfloat16()
    table = torch.full((1, 4), -1, dtype=torch.int32, device=DEV)
    table[0, 3] = N - 1
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    ax.axon_kv_append(cache, 0, x[:, G:2 * G], x[:, 2 * G:], torch.tensor([55], dtype=torch.int32, device=DEV), table, err=err)
    assert torch.equal(k[0, -1, :, 7], x[0, G:2 * G]) and torch.equal(v[0, -1, :, 7], x[0, 2 * G:])
    assert not k[0, -1, :, :7].any() and not k[0, -1, :, 8:].any()
    assert ax.axon_check_error(err) == (0, 0)


def test_captured_and_replayed_on_another_stream(ax):
    c = Case(8, 2, 64, "bf16", [5, 20], [1, 1], per=4)
    rope = ax.axon_rope_table(64, 64, 1e4)
    cache = ax.make_kv_cache(c.k, c.v)
    q, k, v = c.parts()
    out = torch.zeros(2, 8, 64, dtype=c.t, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            ax.axon_kv_append(cache, 1, k, v, c.ctx, c.bt, rope=rope, q=q, q_out=out, err=c.err)
            c.ctx.add_(1)
    torch.cuda.current_stream().wait_stream(s)
    k0 = c.k.clone()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    changed = (c.k != k0).any(-1).any(2)[1]  # [blocks, 16]
    want = torch.zeros_like(changed)
    for b, p in enumerate([5, 20]):
        for i in range(3):
            want[c.table[b, (p + i) // 16], (p + i) % 16] = True
    assert torch.equal(changed, want) and c.ctx.tolist() == [8, 23]
