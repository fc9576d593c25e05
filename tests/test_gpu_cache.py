"""The paged cache's calls on the GPU against the model of their rules (oracle/cache.py):
tables, lengths, counts, status and every written row are equal."""
import numpy as np
import pytest
import torch

from oracle.cache import Model
from paper_2605_13433_amd import hstu, paged
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Both:
    """A cache and its model, filled alike."""

    def __init__(self, pages, P, H, d, slots, cols, layers=1, dtype=torch.bfloat16, ts=True, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.c = paged.Cache(pages, P, H, d, slots, cols, layers, dtype, ts)
        k, v = (torch.randn(self.c.k.shape, generator=g).to(dtype) for _ in range(2))
        self.c.k.copy_(k), self.c.v.copy_(v)
        stamp = None
        if ts:
            stamp = np.zeros((pages, P), np.int64)
            self.c.ts.zero_()
        self.m = Model(k.float().numpy(), v.float().numpy(), stamp, slots, cols)
        self.g, self.dtype = g, dtype

    def extend_write(self, slots, counts, stamps=True):
        c, m = self.c, self.m
        start = c.extend(i32(slots), i32(counts))
        want = m.extend(slots, counts)
        assert start.tolist() == want.tolist()
        counts = np.maximum(counts, 0)
        off = np.concatenate([[0], np.cumsum(counts)])
        T = int(off[-1])
        off_t = torch.tensor(off, dtype=torch.int64, device="cuda")
        ts = torch.randint(1 << 50, (T,), generator=self.g)
        for layer in range(c.layers):
            k, v = (torch.randn(T, c.H, c.d, generator=self.g).to(self.dtype) for _ in range(2))
            t = ts if stamps and layer == c.layers - 1 and c.ts is not None else None
            c.write(layer, k.cuda(), v.cuda(), i32(slots), start, off_t, int(counts.max(initial=0)),
                    None if t is None else t.cuda())
            m.write(layer, k.float().numpy(), v.float().numpy(), slots, want, off,
                    None if t is None else t.numpy())
        return start

    def same(self):
        c, m = self.c, self.m
        torch.cuda.synchronize()
        assert np.array_equal(c.tables.cpu().numpy(), m.tables)
        assert np.array_equal(c.lens.cpu().numpy(), m.lens)
        assert np.array_equal(c.refs.cpu().numpy(), m.refs)
        assert int(c.status) == m.status
        assert np.array_equal(c.k.float().cpu().numpy(), m.k)
        assert np.array_equal(c.v.float().cpu().numpy(), m.v)
        if c.ts is not None:
            assert np.array_equal(c.ts.cpu().numpy(), m.ts)
        m.check()


@pytest.mark.parametrize("seed,P,H,d,layers,dtype,ts", [
    (0, 1, 1, 64, 1, torch.bfloat16, True), (1, 4, 3, 64, 2, torch.bfloat16, True),
    (2, 8, 2, 128, 1, torch.bfloat16, False), (3, 16, 5, 32, 3, torch.float32, True),
    (4, 2, 1, 128, 2, torch.float32, True), (5, 32, 8, 128, 1, torch.bfloat16, True)])
def test_random_calls(seed, P, H, d, layers, dtype, ts):
    rng = np.random.default_rng(seed)
    pages, slots, cols = 60, 9, 8
    b = Both(pages, P, H, d, slots, cols, layers, dtype, ts, seed)
    for step in range(60):
        op = int(rng.integers(6))
        some = rng.integers(-1, slots + 1, int(rng.integers(1, slots + 1)))
        say(f"  step {step} op {op} rows {some.tolist()}")
        if op <= 2:
            b.extend_write(some, rng.integers(-1, 3 * P + 2, len(some)), stamps=bool(rng.integers(2)))
        elif op == 3:
            src = rng.integers(-1, slots + 1, len(some))
            b.c.fork(i32(src), i32(some))
            b.m.fork(src, some)
        elif op == 4:
            b.c.free(i32(some))
            b.m.free(some)
        else:
            assert int(b.c.compact()) == b.m.compact()
        b.same()


def test_beams_are_reordered_at_once():
    b = Both(40, 4, 2, 64, 6, 8)
    b.extend_write([0, 1, 2, 3], [5, 9, 2, 16])
    for src, dst in (([1, 0], [0, 1]), ([3, 2, 1, 0], [0, 1, 2, 3]), ([0, 0, 0], [0, 4, 5]),
                     ([5], [5])):
        b.c.fork(i32(src), i32(dst))
        b.m.fork(src, dst)
        b.same()
    # everyone writes: shared last pages part
    b.extend_write([5, 4, 3, 2, 1, 0], [1, 1, 1, 1, 1, 1])
    b.same()


def test_out_of_pages():
    b = Both(6, 4, 1, 64, 5, 4)
    b.extend_write([0, 1, 2, 3, 4], [8, 12, 8, 1, 0])       # 2 + 3 of 6, then 2 and 1 more
    b.same()
    assert int(b.c.status) == paged.HSTU_CACHE_FULL
    b.extend_write([3, 2], [1, 20])                          # the last page; too few columns
    b.same()
    b.c.free(i32([0, 0, 3]))
    b.m.free([0, 3])
    b.same()
    b.c.clear()
    b.m.tables[:], b.m.lens[:], b.m.refs[:], b.m.status = -1, 0, 0, 0
    b.same()


def test_many_rows_and_pages():
    """More rows than threads, more pages than one round of the search, pages far
    apart in a pool of more than 2^31 bytes."""
    rng = np.random.default_rng(7)
    slots, P, pages, cols = 1500, 2, 70000, 40
    c = paged.Cache(pages, P, 64, 128, slots, cols)          # 2 x 2.3 GB
    assert c.k.numel() * c.k.element_size() > 1 << 31
    m = Model(np.zeros((1, pages, P, 1)), np.zeros((1, pages, P, 1)), None, slots, cols)

    def step(rows, counts):
        start = c.extend(i32(rows), i32(counts))
        assert start.tolist() == m.extend(rows, counts).tolist()
        return start

    step(rng.permutation(slots), rng.integers(0, 60, slots))
    gone = rng.permutation(slots)[:700]
    c.free(i32(gone)), m.free(gone)
    for _ in range(3):
        rows = rng.permutation(slots)[:1300]
        step(rows, rng.integers(0, 30, len(rows)))
    src, dst = rng.integers(0, slots, 1400), rng.permutation(slots)[:1400]
    c.fork(i32(src), i32(dst)), m.fork(src, dst)
    start = step(rng.permutation(slots), np.ones(slots))
    assert np.array_equal(c.tables.cpu().numpy(), m.tables)
    assert np.array_equal(c.lens.cpu().numpy(), m.lens)
    assert np.array_equal(c.refs.cpu().numpy(), m.refs)
    # the longest sequence's rows at the pool's far end move to its front and stay readable
    s = int(np.argmax(m.lens))
    n = int(m.lens[s])
    rows = torch.randn(n, 64, 128, device="cuda", dtype=torch.bfloat16)
    c.free(i32([s])), m.free([s])
    far = torch.nonzero(c.refs == 0).view(-1)[:-(n // P + 2)].int()
    c.refs[far.long()] = 1                                    # the front looks taken
    m.refs[far.cpu().numpy()] = 1
    start = step([s], [n])
    assert m.tables[s, 0] > 60000
    c.write(0, rows, -rows, i32([s]), start, torch.tensor([0, n], device="cuda"), n)
    c.refs[far.long()] = 0
    m.refs[far.cpu().numpy()] = 0
    assert int(c.compact()) == m.compact()
    assert np.array_equal(c.tables.cpu().numpy(), m.tables)
    assert np.array_equal(c.refs.cpu().numpy(), m.refs)
    p = c.tables[s].long()
    x = torch.arange(n, device="cuda")
    assert torch.equal(c.k[0][p[x // P], x % P], rows)
    assert torch.equal(c.v[0][p[x // P], x % P], -rows)


@pytest.mark.parametrize("n,most", [(1, 1), (63, 40), (64, 1), (65, 17), (700, 33), (4500, 5)])
def test_rows_of_every_length(n, most):
    """Batches of one to thousands of rows, of no tokens up to several work-groups' worth,
    in any order of the slots; the second call starts inside pages."""
    rng = np.random.default_rng(n)
    P = 4
    b = Both(n * (2 * most // P + 2), P, 1, 32, n + 9000, 2 * most // P + 2, 2, torch.float32,
             seed=n)
    for _ in range(2):                  # (more slots than the plan keeps in LDS)
        b.extend_write(rng.permutation(n + 9000)[:n] if n < 700 else np.arange(n)[::-1].copy(),
                       rng.integers(0, most + 1, n))
    b.same()


@pytest.mark.parametrize("max_new", [0, 1, 15, 16, 17, 31, 99])
def test_write_stops_at_max_new(max_new):
    b = Both(40, 8, 2, 64, 4, 10)
    counts = np.array([33, 0, 50, 3])
    slots = np.array([2, 0, 3, 1])
    start = b.c.extend(i32(slots), i32(counts))
    want = b.m.extend(slots, counts)
    off = np.concatenate([[0], np.cumsum(counts)])
    k, v = (torch.randn(int(off[-1]), 2, 64, generator=b.g).bfloat16() for _ in range(2))
    ts = torch.arange(int(off[-1])) + 5
    b.c.write(0, k.cuda(), v.cuda(), i32(slots), start, torch.tensor(off, device="cuda"), max_new,
              ts.cuda())
    for r in range(4):                               # the model, a row's first tokens alone
        n = min(int(counts[r]), max_new)
        b.m.write(0, k.float().numpy()[off[r]:], v.float().numpy()[off[r]:], slots[r:r + 1],
                  want[r:r + 1], np.array([0, n]), ts.numpy()[off[r]:])
    b.same()


def test_write_checks_tables_and_offsets_on_the_device():
    """Entries that name no page, starts past the table and offsets past the rows write
    nothing outside; the row behind the last one stays as it was."""
    b = Both(8, 4, 1, 64, 3, 2)
    b.extend_write([0, 1], [3, 8])
    before = b.c.k.clone(), b.c.v.clone()
    rows = torch.ones(6, 1, 64, dtype=torch.bfloat16, device="cuda")
    b.c.tables[2, 0] = 8
    b.c.tables[2, 1] = -5
    b.c.write(0, rows, rows, i32([2, 1, 0]), i32([0, 8, -1]),
              torch.tensor([0, 3, 5, 6], device="cuda"), 8)
    b.c.write(0, rows, rows, i32([7, -1]), i32([0, 0]), torch.tensor([0, 3, 6], device="cuda"), 8)
    b.c.write(0, rows, rows, i32([0]), i32([0]), torch.tensor([6, 99], device="cuda"), 99)
    b.c.write(0, rows, rows, i32([0]), i32([0]), torch.tensor([-4, -2], device="cuda"), 99)
    torch.cuda.synchronize()
    assert torch.equal(b.c.k, before[0]) and torch.equal(b.c.v, before[1])
    # no more than max_new tokens of a row
    b.c.write(0, rows, rows, i32([0]), i32([0]), torch.tensor([0, 2], device="cuda"), 2)
    p = int(b.c.tables[0, 0])
    assert (b.c.k[0, p, :2] == 1).all() and torch.equal(b.c.k[0, p, 2:], before[0][0, p, 2:])


def test_graph_replays():
    """A beam step captured once and replayed, eager calls in between."""
    b = Both(64, 4, 2, 64, 12, 8, layers=2)
    b.extend_write([0, 1, 2], [6, 9, 11])
    c = b.c
    src, dst = i32([0, 0, 1, 2, 2, 2]), i32([3, 4, 5, 6, 7, 8])
    counts, off = i32([1] * 6), torch.arange(7, device="cuda")
    k = torch.randn(2, 6, 2, 64, device="cuda").bfloat16()
    ts = torch.arange(6, device="cuda")
    start = torch.empty(6, dtype=torch.int32, device="cuda")

    def step():
        c.free(dst)
        c.fork(src, dst)
        c.extend(dst, counts, start=start)
        c.write(0, k[0], k[1], dst, start, off, 1, ts)
        c.write(1, k[1], k[0], dst, start, off, 1)

    def state():
        torch.cuda.synchronize()
        return [t.clone() for t in (c.k, c.v, c.ts, c.tables, c.lens, c.refs, start, c.status)]

    step()
    want = state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        c.k[:, c.tables[3, -1].clamp(min=0).long()].sum().item()      # eager work between
        graph.replay()
        for a, w in zip(state(), want):
            assert torch.equal(a, w)
        c.free(i32([9, 10]))


def test_refusals_in_python():
    c = paged.Cache(8, 4, 2, 64, 3, 2)
    ok = i32([0, 1])
    with pytest.raises(ValueError, match="int32"):
        c.extend(ok.long(), ok)
    with pytest.raises(ValueError, match="is on cpu"):
        c.free(ok.cpu())
    with pytest.raises(ValueError, match="shape"):
        c.extend(ok, i32([1]))
    with pytest.raises(hstu.HstuError, match="3 slots"):
        c.free(i32([0, 1, 2, 0]))
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    off = torch.arange(3, device="cuda")
    start = c.extend(ok, ok)
    with pytest.raises(ValueError, match="shape"):
        c.write(0, k[:, :1], k, ok, start, off, 1)
    with pytest.raises(ValueError, match="k must be"):
        c.write(0, k.float(), k, ok, start, off, 1)
    with pytest.raises(ValueError, match="contiguous"):
        c.write(0, k.transpose(0, 1).contiguous().transpose(0, 1), k, ok, start, off, 1)
    with pytest.raises(hstu.HstuError, match="layer = 1"):
        c.write(1, k, k, ok, start, off, 1)
    with pytest.raises(ValueError, match="without a window"):
        paged.DecodePlan(c, 2, 8, sinks=1)
    with pytest.raises(ValueError, match="pos_w has shape"):
        paged.DecodePlan(c, 2, 8, pos_w=torch.zeros(2, 14, device="cuda"))
    plan = paged.DecodePlan(c, 2, 8)
    with pytest.raises(ValueError, match="3 slots for"):
        plan.forward(k, k.view(2, -1), i32([0, 1, 2]))
    with pytest.raises(ValueError, match="u has shape"):
        plan.forward(k, k, ok)
