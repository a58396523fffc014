"""Attention over shared prefixes (axon_attn_shared) against attention in 64 bits, one query at a time (kv_model.attention).

Every slot of the pools that no query of a case may see holds NaN, and every table entry that the mask hides is -1.

Tolerances, as for axon_attn_decode: inputs are exact; scores are fp32 sums of 128 products at most, of magnitude sum |q k| *
scale < 30, off by < 128 * 2^-24 * 30 = 2.3e-4, twice that on a probability's ratio: an output moves by 5e-4 max |v| at
most (the joins of parts, a few 2^-24, among it), and lse by 5e-4; the output's rounding adds half a unit, doubled here."""
import numpy as np
import pytest

import kv_model as km

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ULP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -10}
DEV = "cuda"


@pytest.fixture(scope="module")
def ax():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


@pytest.fixture(autouse=True)
def small_cases_share_too(monkeypatch):
    """Sharing saves too little in cases of this size to be taken by itself."""
    monkeypatch.setenv("AXON_SHARED_MIN_BYTES", "0")


class Case:
    """groups: (tokens whose whole blocks are shared, positions of the rows' queries, None: idle; grouped or loose)."""

    def __init__(self, H, G, d, dtype, groups, window=0, sinks=0, seed=0, layers=2, layer=1, said=None):
        r = np.random.default_rng(seed)
        self.H, self.G, self.d, self.dtype, self.window, self.sinks, self.layer = H, G, d, dtype, window, sinks, layer
        t = TYPES[dtype]
        self.pos = [-1 if p is None else p for _, rows in groups for p in rows]
        B = len(self.pos)
        self.per = max(1, max(p // 16 + 1 for p in self.pos))
        N = sum(pre // 16 for pre, _ in groups) + B * self.per + 3
        k = torch.full((layers, N, G, 16, d), float("nan"), dtype=t)
        v = k.clone()
        perm = list(r.permutation(N))
        self.table = np.full((B, self.per), -1, dtype=np.int32)
        self.keys, self.values = [], []
        make = lambda n: torch.from_numpy(r.standard_normal((n, G, d))).to(t)  # noqa: E731
        row = 0
        for pre, rows in groups:
            live = [p for p in rows if p is not None]
            whole = pre // 16
            longest = max([p + 1 for p in live], default=0)
            first = min([max(0, p - window + 1) if window else 0 for p in live], default=0)
            sk, sv = make(whole * 16), make(whole * 16)
            blocks = []
            for j in range(min(whole, -(-longest // 16))):
                if window and (j + 1) * 16 <= first and j * 16 >= sinks:
                    blocks.append(-1)  # hidden from all
                    continue
                b = perm.pop()
                blocks.append(b)
                # what the longest row sees; the window may hide more, which the mask of every row covers
                hi = min(longest, j * 16 + 16) - j * 16
                k[layer, b, :, :hi] = sk[j * 16:j * 16 + hi].transpose(0, 1)
                v[layer, b, :, :hi] = sv[j * 16:j * 16 + hi].transpose(0, 1)
            for p in rows:
                if p is None:
                    self.keys.append(np.zeros((0, G, d)))
                    self.values.append(np.zeros((0, G, d)))
                    row += 1
                    continue
                n = p + 1
                self.table[row, :len(blocks)] = blocks[:self.per]
                ok, ov = make(max(0, n - whole * 16)), make(max(0, n - whole * 16))
                lo = max(0, n - window) if window else 0
                for j in range(whole, -(-n // 16)):
                    if window and (j + 1) * 16 <= lo and j * 16 >= sinks:
                        continue
                    b = perm.pop()
                    self.table[row, j] = b
                    at, hi = j * 16 - whole * 16, min(n, j * 16 + 16) - j * 16
                    k[layer, b, :, :hi] = ok[at:at + hi].transpose(0, 1)
                    v[layer, b, :, :hi] = ov[at:at + hi].transpose(0, 1)
                self.keys.append(torch.cat([sk, ok])[:n].double().numpy())
                self.values.append(torch.cat([sv, ov])[:n].double().numpy())
                row += 1
        self.k, self.v = k.to(DEV), v.to(DEV)
        self.q = torch.from_numpy(r.standard_normal((B, H, d)) * 1.6).to(t).to(DEV)
        self.ctx = torch.tensor(self.pos, dtype=torch.int32, device=DEV)
        self.bt = torch.from_numpy(self.table).to(DEV)
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum([len(g[1]) for g in groups])]), dtype=torch.int32, device=DEV)
        self.prefix = torch.tensor([g[0] for g in groups] if said is None else said, dtype=torch.int32, device=DEV)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)

    def reference(self, rows, scale=None):
        q = self.q.double().cpu().numpy()
        o, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
        for b in rows:
            if self.pos[b] >= 0:
                o[b], lse[b] = km.attention(q[b], self.keys[b], self.values[b], self.pos[b], self.window, self.sinks, scale)
        return o, lse


def run(ax, c, q=None, out=None, work=None, **kw):
    cache = ax.make_kv_cache(c.k, c.v)
    work = ax.make_shared_workspace(cache, len(c.pos), c.H) if work is None else work
    q = c.q if q is None else q
    out = torch.full_like(c.q, float("nan")) if out is None else out
    lse = torch.full((len(c.pos), c.H), float("nan"), device=DEV)
    ax.axon_attn_shared(cache, c.layer, q, c.ctx, c.offsets, c.prefix, out, work, c.bt, window=c.window, sinks=c.sinks, lse=lse,
                        err=c.err, **kw)
    return out, lse


def check(ax, c, rows=None, err=(0, 0), **kw):
    out, lse = run(ax, c, **kw)
    rows = range(len(c.pos)) if rows is None else rows
    rows = list(rows)
    want, wlse = c.reference(rows, kw.get("scale"))
    got, lse = out.double().cpu().numpy()[rows], lse.double().cpu().numpy()[rows]
    want, wlse = want[rows], wlse[rows]
    assert np.isfinite(got).all()
    vmax = max([np.abs(v).max() for v in c.values if v.size], default=0.0)
    off = np.abs(got - want) - ULP[c.dtype] * np.abs(want)
    assert off.max(initial=0.0) <= 5e-4 * vmax, f"off by {off.max():.3e}, {5e-4 * vmax:.3e} allowed"
    empty = np.isinf(wlse)
    assert np.array_equal(np.isneginf(lse), empty)
    assert np.abs(lse[~empty] - wlse[~empty]).max(initial=0.0) <= 5e-4
    assert ax.axon_check_error(c.err) == err


HEADS = [(14, 2, 64), (32, 8, 128), (9, 3, 64), (4, 4, 128), (10, 1, 128), (16, 1, 64), (40, 8, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,d", HEADS)
def test_groups_of_all_kinds(ax, H, G, d, dtype):
    groups = [(700, [700, 735, 704, 1000]),           # samples that have parted
              (0, [50]), (256, [255, 255]),           # all of both rows in common
              (129, [128, 140, 300]), (515, []),      # a prefix that ends in a block; no rows
              (2000, [400, 17, 401]),                 # a prefix that is longer than the rows
              (64, [90, 91]), (1500, [None, 1600, None, 1499, 1510])]
    check(ax, Case(H, G, d, dtype, groups, seed=H * d))


@pytest.mark.parametrize("rows", [2, 9, 31, 32, 33, 63, 64, 65, 130])
@pytest.mark.parametrize("H,G,d", [(32, 8, 128), (14, 2, 64), (3, 3, 64)])
def test_group_sizes(ax, rows, H, G, d):
    r = np.random.default_rng(rows)
    check(ax, Case(H, G, d, "bf16", [(400, [int(p) for p in r.integers(383, 520, rows)])], seed=rows))


@pytest.mark.parametrize("blocks", [7, 8, 9, 15, 16, 17, 24, 65])
def test_prefix_lengths(ax, blocks):
    n = 16 * blocks
    check(ax, Case(8, 2, 128, "fp16", [(n, [n - 1, n, n + 15]), (n + 15, [n + 16, n + 40])], seed=blocks))


@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 0), (300, 4), (301, 33), (512, 16), (900, 5), (2000, 4), (299, 1000)])
@pytest.mark.parametrize("H,G,d", [(6, 2, 128), (12, 1, 64)])
def test_window_and_sinks(ax, H, G, d, window, sinks):
    groups = [(1000, [1000, 1010, 1100, 1250]), (300, [305, 700]), (800, [799, 803, None, 805])]
    check(ax, Case(H, G, d, "bf16", groups, window, sinks, seed=window))


def test_a_long_prefix_over_all_multiprocessors(ax):
    c = Case(14, 2, 64, "bf16", [(30000, [30000, 30005, 30100])], seed=1, layers=1, layer=0)
    check(ax, c)
    c = Case(8, 8, 128, "fp16", [(9000, [9001 + 3 * i for i in range(20)])], seed=2, layers=1, layer=0)
    check(ax, c, rows=[0, 7, 19])


def test_many_rows_and_groups(ax):
    r = np.random.default_rng(3)
    groups = [(int(p), [int(p) + int(x) for x in r.integers(-20, 60, n)])
              for p, n in zip(r.integers(130, 700, 300), r.integers(1, 9, 300))]
    c = Case(8, 2, 64, "bf16", groups, seed=4, layers=1, layer=0)
    check(ax, c, rows=r.permutation(len(c.pos))[:200])


def test_most_rows_and_groups(ax):
    c = Case(2, 1, 64, "bf16", [(160, [165, 170])] * 1024, seed=5, layers=1, layer=0)
    check(ax, c, rows=[0, 1, 1000, 2046, 2047])
    c = Case(2, 1, 64, "bf16", [(160, [165 + i % 7 for i in range(2048)])], seed=5, layers=1, layer=0)
    check(ax, c, rows=[0, 63, 64, 127, 128, 2047])


def test_scores_that_grow_along_the_prefix(ax):
    """Maxima that rise step by step, and keys that outweigh everything before them."""
    c = Case(8, 2, 128, "bf16", [(2048, [2050, 2100, 2047])], seed=6, layers=1, layer=0)
    for b in range(3):
        grow = np.linspace(0.2, 5.0, c.keys[b].shape[0])[:, None, None]
        keys = torch.from_numpy(c.keys[b] * grow).to(TYPES["bf16"])
        for j in range(-(-keys.shape[0] // 16)):
            part = keys[j * 16:j * 16 + 16]
            c.k[0, int(c.table[b, j]), :, :part.shape[0]] = part.transpose(0, 1).to(DEV)
    for b in range(3):  # (the blocks in common hold what was written last)
        held = c.k[0][c.bt[b].long()].transpose(1, 2).reshape(-1, c.G, c.d)
        c.keys[b] = held[:c.pos[b] + 1].double().cpu().numpy()
    out, lse = run(ax, c)
    # scores reach 5 times those of the tolerance above
    want, wlse = c.reference(range(3))
    vmax = max(np.abs(v).max() for v in c.values)
    off = np.abs(out.double().cpu().numpy() - want) - ULP["bf16"] * np.abs(want)
    assert off.max() <= 2.5e-3 * vmax
    assert np.abs(lse.double().cpu().numpy() - wlse).max() <= 2.5e-3


def test_strides_scale_and_rows_outside_groups(ax):
    c = Case(8, 2, 64, "bf16", [(300, [310, 320, 330]), (200, [250, 260]), (150, [170, 180, 181])], seed=7)
    wide = torch.full((8, 11, 64 + 24), float("nan"), dtype=c.q.dtype, device=DEV)
    q, out = wide[:, 1:9, 8:72], torch.full((8, 2, 8, 64), float("nan"), dtype=c.q.dtype, device=DEV)[:, 1]
    q.copy_(c.q)
    check(ax, c, q=q, out=out, scale=0.21)
    c.offsets = c.offsets[1:3].clone()  # the first three rows and the last three belong to no group
    c.prefix = c.prefix[1:2].clone()
    check(ax, c)


def test_idle_rows_first_and_alone(ax):
    c = Case(8, 2, 64, "bf16", [(300, [None, None, 310, 320]), (200, [None, None]), (400, [None, 410]), (0, [None])], seed=8)
    check(ax, c)


def test_reported_faults(ax):
    def case():
        return Case(8, 2, 64, "bf16", [(300, [310, 320, 330]), (200, [250, 260])], seed=9)
    for offsets in ([0, 4, 3], [-1, 3, 5], [0, 3, 6], [3, 0, 5], [0, 1 << 30, 5]):
        c = case()
        c.offsets = torch.tensor(offsets, dtype=torch.int32, device=DEV)
        check(ax, c, err=(8, 16))  # nothing shared, every row right
    c = case()
    c.prefix[0] = -5
    check(ax, c, err=(8, 4))
    c = case()
    c.bt[0, 3] = c.k.shape[1]  # in the first group's common part
    check(ax, c, rows=[3, 4], err=(8, 2))
    out, _ = run(ax, c)
    assert torch.isfinite(out).all() and ax.axon_check_error(c.err)[1] == 2
    c = case()
    c.ctx[1] = c.per * 16
    c.pos[1] = -1
    check(ax, c, err=(8, 4))


def test_one_workspace_for_many_shapes_and_the_plain_form(ax):
    big = Case(32, 8, 128, "bf16", [(900, [910 + i for i in range(40)])], seed=10)
    cache = ax.make_kv_cache(big.k, big.v)
    work = ax.make_shared_workspace(cache, 64, 32)
    small = Case(32, 8, 128, "bf16", [(200, [210, 220, 300]), (700, [701, 703])], seed=11)
    for c in (big, small, big, small):
        check(ax, c, work=work)
        sc = ax.make_kv_cache(c.k, c.v)
        a, b = torch.empty_like(c.q), torch.empty_like(c.q)
        ax.axon_attn_decode(sc, c.layer, c.q, c.ctx, a, work, block_table=c.bt)
        ax.axon_attn_decode(sc, c.layer, c.q, c.ctx, b, ax.make_attn_workspace(sc, len(c.pos), 32), block_table=c.bt)
        assert torch.equal(a, b)


def test_same_bits_every_time_captured_and_on_another_stream(ax):
    c = Case(32, 8, 128, "bf16", [(900, [910 + i for i in range(13)]), (300, [301, 350])], seed=12)
    cache = ax.make_kv_cache(c.k, c.v)
    work = ax.make_shared_workspace(cache, len(c.pos), 32)
    first, lse0 = run(ax, c, work=work)
    out, lse = torch.empty_like(c.q), torch.empty_like(lse0)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            for _ in range(3):
                ax.axon_attn_shared(cache, c.layer, c.q, c.ctx, c.offsets, c.prefix, out, work, c.bt, lse=lse)
    torch.cuda.current_stream().wait_stream(s)
    for _ in range(4):
        out.zero_()
        g.replay()
        assert torch.equal(out, first) and torch.equal(lse, lse0)
    c.ctx.sub_(30)  # shorter rows by the time of the replay: the blocks in common are found anew
    c.pos = [p - 30 for p in c.pos]
    c.keys, c.values = [k[:-30] for k in c.keys], [v[:-30] for v in c.values]
    g.replay()
    want, _ = c.reference(range(len(c.pos)))
    off = np.abs(out.double().cpu().numpy() - want) - ULP["bf16"] * np.abs(want)
    assert off.max() <= 5e-4 * max(np.abs(v).max() for v in c.values)


def test_where_sharing_does_not_pay_by_itself(ax, monkeypatch):
    """The library's own limit: no prefix pass for tables so narrow (alone), none for rows so short (found on the device)."""
    monkeypatch.delenv("AXON_SHARED_MIN_BYTES")
    groups = [(300, [310, 320, 330]), (200, [250, None]), (400, [470, 410, 399, 500])]
    for per in (0, 4096):
        c = Case(32, 8, 128, "bf16", groups, seed=13)
        if per:
            c.bt = torch.nn.functional.pad(c.bt, (0, per - c.per), value=-1)
        check(ax, c)
        plain = torch.empty_like(c.q)
        cache = ax.make_kv_cache(c.k, c.v)
        ax.axon_attn_decode(cache, c.layer, c.q, c.ctx, plain, ax.make_attn_workspace(cache, len(c.pos), 32), block_table=c.bt)
        assert torch.equal(run(ax, c)[0], plain)
    c.offsets[1] = 100
    check(ax, c, err=(8, 16))
    c = Case(32, 8, 128, "bf16", groups, seed=13)
    c.offsets[1], c.prefix[2] = -1, -7
    check(ax, c, err=(8, 20))


@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 4)])
def test_where_it_does(ax, monkeypatch, window, sinks):
    """40 rows on 4096 tokens, by the library's own limit, against the one-token form."""
    monkeypatch.delenv("AXON_SHARED_MIN_BYTES")
    r = np.random.default_rng(14)
    B, G, d, per, whole = 43, 8, 128, 300, 256
    N = whole + B * (per - whole)
    g = torch.Generator(device=DEV)
    g.manual_seed(14)
    k, v = (torch.empty(1, N, G, 16, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    q = torch.empty(B, 32, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g) * 1.6
    table = np.concatenate([np.tile(np.arange(whole), (B, 1)), whole + np.arange(B * (per - whole)).reshape(B, -1)], 1)
    bt = torch.from_numpy(table.astype(np.int32)).to(DEV)
    ctx = torch.from_numpy(r.integers(whole * 16, per * 16, B).astype(np.int32)).to(DEV)
    cache = ax.make_kv_cache(k, v)
    work = ax.make_shared_workspace(cache, B, 32)
    a, b = torch.empty_like(q), torch.empty_like(q)
    la, lb = torch.empty(B, 32, device=DEV), torch.empty(B, 32, device=DEV)
    offsets, prefix = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 40, 43], [4096, 16]))
    ax.axon_attn_shared(cache, 0, q, ctx, offsets, prefix, a, work, bt, window=window, sinks=sinks, lse=la)
    ax.axon_attn_decode(cache, 0, q, ctx, b, work, block_table=bt, window=window, sinks=sinks, lse=lb)
    assert not torch.equal(a, b)  # other sums: the prefix pass ran
    vmax = float(v.abs().max())
    assert ((a.double() - b.double()).abs() <= 5e-4 * vmax + 2.0 ** -7 * b.double().abs()).all()
    assert float((la - lb).abs().max()) <= 5e-4


def test_thousands_of_calls_in_a_row(ax):
    """Three states in turn, one tile and two per group, each call with an output of its own: the same bits every time."""
    cases = [Case(32, 8, 128, t, [(g, [g + 20 + 3 * j for j in range(w)]) for g, w in groups], seed=20 + n, layers=1, layer=0)
             for n, (t, groups) in enumerate([("fp16", [(2176, 4), (900, 3), (1500, 4), (700, 2)]),
                                              ("bf16", [(1700, 40), (333, 5), (640, 33), (1040, 4)]),
                                              ("fp16", [(1160, 4), (520, 4), (1290, 3)])])]
    state, n = [], 1200
    for c in cases:
        cache = ax.make_kv_cache(c.k, c.v)
        work = ax.make_shared_workspace(cache, len(c.pos), 32)
        state.append((c, cache, work, torch.zeros(n, *c.q.shape, dtype=c.q.dtype, device=DEV), run(ax, c, work=work)[0]))
    torch.cuda.synchronize()
    for i in range(3 * n):
        c, cache, work, outs, _ = state[i % 3]
        ax.axon_attn_shared(cache, 0, c.q, c.ctx, c.offsets, c.prefix, outs[i // 3], work, c.bt)
    for _, _, _, outs, want in state:
        assert (outs == want).all()


@pytest.mark.parametrize("common,own", [(160, 5000), (6000, 2), (6000, 5000), (1024, 300)])
def test_how_the_multiprocessors_are_shared_out(ax, common, own):
    """Most of the work in the rows' own parts, in the common ones, in both, and little of either."""
    check(ax, Case(12, 2, 128, "bf16", [(common, [common + own + 7 * j for j in range(5)])], seed=common + own, layers=1, layer=0))


def test_two_calls_at_once(ax):
    """On two streams with a workspace each: CTAs of the one come where the other expects its own. The same bits as alone."""
    cases = [Case(32, 8, 128, "bf16", [(2000, [2020 + 300 * j for j in range(8)]), (700, [720, 731, 2500])], seed=61, layers=1, layer=0),
             Case(14, 2, 64, "fp16", [(5000, [5010 + j for j in range(20)])], seed=62, layers=1, layer=0)]
    n, state = 300, []
    for c in cases:
        cache = ax.make_kv_cache(c.k, c.v)
        work = ax.make_shared_workspace(cache, len(c.pos), c.q.shape[1])
        want = run(ax, c, work=work)[0]
        state.append((c, cache, work, torch.zeros(n, *c.q.shape, dtype=c.q.dtype, device=DEV), want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(n):
        for c, cache, work, outs, _, stream in state:
            ax.axon_attn_shared(cache, 0, c.q, c.ctx, c.offsets, c.prefix, outs[i], work, c.bt, stream=stream)
    torch.cuda.synchronize()
    for _, _, _, outs, want, _ in state:
        assert (outs == want).all()
