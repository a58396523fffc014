"""Blocks of a paged key/value cache (copy, fork, release, reserve, compact) against
plain bookkeeping on host lists (kv_model.Pages): tables, lengths, counts and contents,
bit for bit."""
import numpy as np
import pytest

import kv_model as km

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


class Cache:
    """A cache on the device and its model: rows of `lens` tokens in shuffled blocks, contents random."""

    def __init__(self, ax, lens, N, P, shape=(2, 2, 64), dtype=torch.bfloat16, seed=0, share=()):
        L, G, d = shape
        r = np.random.default_rng(seed)
        table, refs = np.full((len(lens), P), -1), np.zeros(N, dtype=int)
        perm, at = r.permutation(N), 0
        for b, n in enumerate(lens):
            need = -(-n // 16)
            table[b, :need] = perm[at:at + need]
            refs[perm[at:at + need]] += 1
            at += need
        for a, b in share:  # row b starts with row a's first block
            refs[table[b, 0]] -= 1
            table[b, 0] = table[a, 0]
            refs[table[a, 0]] += 1
        self.ax, self.model = ax, km.Pages(table, lens, refs)
        self.k, self.v = (torch.randn(L, N, G, 16, d, device="cuda").to(dtype) for _ in range(2))
        self.k0, self.v0 = self.k.clone(), self.v.clone()
        self.table, self.ctx, self.refs = (torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
                                           for x in (table, lens, refs))
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.cache = ax.make_kv_cache(self.k, self.v)
        self.seqs = ax.make_kv_seqs(self.table, self.ctx, self.refs)
        self.work = ax.make_kv_workspace(self.cache, self.seqs)
        self.work.fill_(0xA5)  # may hold anything

    def ints(self, v):
        return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda")

    def release(self, rows, window=0, sinks=0):
        self.ax.axon_kv_release(self.cache, self.seqs, self.ints(rows), window=window, sinks=sinks, err=self.err)
        self.model.release(rows, window, sinks)

    def reserve(self, rows, new):
        self.ax.axon_kv_reserve(self.cache, self.seqs, self.ints(rows), self.ints(new), self.work, err=self.err)
        self.model.reserve(rows, new)

    def fork(self, src, dst):
        self.ax.axon_kv_fork(self.cache, self.seqs, self.ints(src), self.ints(dst), self.work, err=self.err)
        self.model.fork(src, dst)

    def compact(self):
        moved = torch.full((len(self.model.refs),), -7, dtype=torch.int32, device="cuda")
        live = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        self.ax.axon_kv_compact(self.cache, self.seqs, self.work, moved=moved, live=live, err=self.err)
        m, n = self.model.compact()
        assert np.array_equal(moved.cpu().numpy(), m) and int(live) == n

    def check(self, bits=0):
        m = self.model
        for name in ("table", "ctx", "refs"):
            assert np.array_equal(getattr(self, name).cpu().numpy(), getattr(m, name)), name
        # every block in use holds what its tag says; the counts are the table's
        used = np.nonzero(m.refs)[0]
        tag = torch.from_numpy(m.tag[used]).cuda()
        at = torch.from_numpy(used).cuda()
        assert torch.equal(self.k[:, at], self.k0[:, tag]) and torch.equal(self.v[:, at], self.v0[:, tag])
        assert np.array_equal(np.bincount(m.table[m.table >= 0], minlength=len(m.refs)), m.refs)
        want = self.ax.AXON_ERR_DEVICE_CHECK if bits else 0
        assert self.ax.axon_check_error(self.err) == (want, bits)


SHAPES = [((2, 2, 64), torch.bfloat16), ((1, 1, 64), torch.float16), ((3, 8, 128), torch.float16), ((2, 3, 64), torch.float32)]


@pytest.mark.parametrize("shape,dtype", SHAPES)
def test_fork_samples_of_one_prompt(ax, shape, dtype):
    c = Cache(ax, [37, 0, 0, 0, 50], 40, 6, shape, dtype)
    c.fork([0, 0, 0], [1, 2, 3])
    c.check()
    c.fork([0, 0, 0], [1, 2, 3])  # again: the copies give their block back and take it
    c.check()


@pytest.mark.parametrize("lens", [[33, 33, 33, 33], [32, 48, 1, 15], [0, 16, 17, 31], [5, 5, 5, 5]])
@pytest.mark.parametrize("src", [[1, 0, 3, 2], [0, 0, 0, 0], [3, 3, 2, 1], [1, 2, 3, 0], [0, 1, 2, 3]])
def test_fork_permutes_rows_as_they_were(ax, lens, src):
    c = Cache(ax, lens, 24, 5, share=[(0, 2)] if lens[0] >= 16 and lens[2] >= 16 else [])
    c.fork(src, [0, 1, 2, 3])
    c.check()


def test_fork_over_longer_rows_and_reserved_blocks(ax):
    c = Cache(ax, [20, 90, 0], 30, 8)
    c.reserve([0, 1], [60, 3])
    c.check()
    c.fork([0, 1], [1, 2])
    c.check()


def test_fork_when_the_pool_runs_out(ax):
    c = Cache(ax, [20, 0, 0, 0], 4, 3)  # two free blocks for three copies
    c.fork([0, 0, 0], [3, 1, 2])
    c.check(bits=32)
    assert c.model.short and c.model.ctx[2] == 16


def test_fork_takes_blocks_that_it_gives_back(ax):
    c = Cache(ax, [20, 33], 5, 3)  # no free block: the row's own three come back
    c.fork([0], [1])
    c.check()


@pytest.mark.parametrize("src,dst,bits", [([0, 0], [1, 1], 16), ([0, 5], [1, 2], 16), ([0, 1], [2, -1], 16), ([3, 0], [1, 2], 4)])
def test_fork_reports_what_it_skips(ax, src, dst, bits):
    c = Cache(ax, [20, 3, 0, 0], 12, 3)
    if bits == 4:
        c.ctx[3] = 49  # past the row
    ok = {16: slice(0, 1), 4: slice(1, 2)}[bits]
    c.ax.axon_kv_fork(c.cache, c.seqs, c.ints(src), c.ints(dst), c.work, err=c.err)
    if bits == 4:
        c.ctx[3] = 0
    c.model.fork(src[ok], dst[ok])
    c.check(bits)


def test_release_whole_rows(ax):
    c = Cache(ax, [37, 16, 0, 100, 5], 40, 8, share=[(0, 3)])
    c.release([3, 2, 0])
    c.check()
    c.release([3, 3, 1])  # rows that hold nothing, and one named twice
    c.check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (17, 1), (20, 16), (33, 17), (64, 4), (5, 1000), (10000, 4), (9, 2 ** 31 - 1),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
def test_release_what_a_window_has_passed(ax, window, sinks):
    lens = [0, 1, 16, 31, 32, 33, 47, 48, 64, 65, 127, 128, 129, 200]
    c = Cache(ax, lens, 100, 14)
    c.release(range(len(lens)), window, sinks)
    c.check()
    c.reserve(range(len(lens)), [1] * len(lens))
    c.check()


def test_release_a_wide_row(ax):
    """More entries than the launch covers at once."""
    c = Cache(ax, [100, 1200000], 75100, 75010, (1, 1, 64))
    c.release([1, 0], 600000, 20)
    c.check()
    c.release([1])
    c.check()


def test_release_reports(ax):
    c = Cache(ax, [37, 16], 8, 4)
    c.ax.axon_kv_release(c.cache, c.seqs, c.ints([2, 1]), err=c.err)
    c.model.release([1])
    c.check(16)
    c.ctx[0] = 65
    c.ax.axon_kv_release(c.cache, c.seqs, c.ints([0]), window=4, err=c.err)
    c.ctx[0] = 37
    c.check(4)
    c.table[0, 3] = 8
    c.ax.axon_kv_release(c.cache, c.seqs, c.ints([0]), err=c.err)
    c.model.release([0])
    c.check(2)


@pytest.mark.parametrize("new", [[0, 0, 0, 0], [1, 1, 1, 1], [16, 15, 17, 0], [40, 3, 33, 60]])
def test_reserve(ax, new):
    c = Cache(ax, [0, 1, 16, 31], 60, 9)
    c.reserve([2, 0, 3, 1], new)
    c.check()
    c.reserve([1, 3], [70, 50])  # some of it is there already
    c.check()


def test_reserve_when_the_pool_runs_out(ax):
    c = Cache(ax, [5, 5, 5], 8, 5)
    c.reserve([1, 0, 2], [30, 30, 30])  # five free blocks for six
    c.check(32)


def test_reserve_reports(ax):
    c = Cache(ax, [5, 40, 16, 7], 30, 5)
    c.ax.axon_kv_reserve(c.cache, c.seqs, c.ints([0, 1, 0]), c.ints([20, 41, 20]), c.work, err=c.err)
    c.model.reserve([0], [20])
    c.check(16 | 4)  # row 1 would pass its end, row 0 comes twice
    c.ax.axon_kv_reserve(c.cache, c.seqs, c.ints([-1, 4, 2]), c.ints([1, 1, -1]), c.work, err=c.err)
    c.check(16 | 4)
    # a row with a block behind a hole
    free = int(np.nonzero(c.model.refs == 0)[0][0])
    c.table[3, 2], c.refs[free] = free, 1
    c.model.table[3, 2], c.model.refs[free] = free, 1
    c.ax.axon_kv_reserve(c.cache, c.seqs, c.ints([3]), c.ints([40]), c.work, err=c.err)
    c.check(16)


@pytest.mark.parametrize("N,lens", [(40, [37, 16, 100, 5]), (40, []), (1, [3]), (9000, [3000, 50000, 16, 0, 17]),
                                    (4096, [40000, 24000]), (4097, [16, 65000]), (14, [100, 70, 30])])
@pytest.mark.parametrize("shape,dtype", SHAPES[:3])
def test_compact(ax, N, lens, shape, dtype):
    if N > 1000 and shape[1] > 2:
        pytest.skip("one shape is enough for large pools")
    lens = lens or [0]
    c = Cache(ax, lens, N, max(2, max(-(-n // 16) for n in lens)), shape, dtype, seed=N)
    c.compact()
    c.check()
    c.compact()  # nothing is left to move
    c.check()


def test_compact_shared_blocks_and_many_rows(ax):
    r = np.random.default_rng(5)
    lens = [int(x) for x in r.integers(1, 200, 120)]
    c = Cache(ax, lens, 3000, 14, share=[(a, a + 1) for a in range(0, 118, 3)], seed=5)
    c.release(range(0, 120, 2))
    c.compact()
    c.check()


def test_compact_reports_entries_that_nothing_counts(ax):
    c = Cache(ax, [20, 30], 20, 4)
    high = max(int(b) for b in np.nonzero(c.model.refs == 0)[0])
    c.table[1, 3] = high
    c.ax.axon_kv_compact(c.cache, c.seqs, c.work, err=c.err)
    assert int(c.table[1, 3]) == high
    c.table[1, 3] = -1
    c.model.compact()
    c.check(2)


def test_copy_blocks(ax):
    c = Cache(ax, [0], 50, 2, (3, 2, 128))
    src, dst = [3, 3, 49, 0, 50, 7, -1], [10, 11, 12, 13, 14, 50, 15]
    c.ax.axon_kv_copy_blocks(c.cache, c.ints(src), c.ints(dst), err=c.err)
    want = c.k0.clone()
    want[:, [10, 11, 12, 13]] = c.k0[:, [3, 3, 49, 0]]
    assert torch.equal(c.k, want)
    c.v0[:, [10, 11, 12, 13]] = c.v0[:, [3, 3, 49, 0]]
    assert torch.equal(c.v, c.v0)
    assert ax.axon_check_error(c.err) == (ax.AXON_ERR_DEVICE_CHECK, 2)


@pytest.mark.parametrize("seed", range(6))
def test_a_life_of_a_cache(ax, seed):
    """Calls one after another without waiting, on pools of one and of several counting chunks."""
    r = np.random.default_rng(100 + seed)
    R, P = 24, 20
    N = [160, 5000][seed % 2]
    lens = [int(x) for x in r.integers(0, 60, R)]
    c = Cache(ax, lens, N, P, seed=seed, share=[(a, a + 1) for a in range(0, R - 1, 5) if lens[a] >= 16 and lens[a + 1] >= 16])
    short = 0
    for _ in range(12):
        kind = r.integers(0, 4)
        rows = [int(x) for x in r.permutation(R)[:r.integers(1, R)]]
        if kind == 0:
            c.release(rows[:3])
        elif kind == 1:
            c.release(rows, window=int(r.integers(1, 40)), sinks=int(r.integers(0, 20)))
        elif kind == 2:
            new = [int(x) for x in r.integers(0, 40, len(rows))]
            new = [min(m, P * 16 - int(c.model.ctx[i])) for m, i in zip(new, rows)]
            c.reserve(rows, new)
            if not c.model.short:  # the tokens are appended
                for m, i in zip(new, rows):
                    c.model.ctx[i] += m
                    c.ctx[i] += m
        elif kind == 3 and not c.model.short:
            n = max(1, len(rows) // 2)
            c.fork(rows[:n], rows[-n:])
        if kind != 1:
            c.compact()
        short |= c.model.short
        if short:
            break
    c.check(32 if short else 0)
