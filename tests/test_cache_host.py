"""The paged cache on the host: the index arithmetic of its kernels (compiled here by
the C++ compiler) against brute force and the bounds of the buffers, the model of its
rules against its own invariants, and the refusals of the C ABI (rejected before the
library touches a device)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle.cache import Model
from oracle.window import seen
from paper_2605_13433_amd import hstu, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = """
#include "cache_index.h"
using namespace hstu;
extern "C" {
int seen_list(int len, int window, int sinks, int *out, int most) {
  const Seen s = seen_by_last(len, window, sinks);
  for (int x = 0; x < s.count && x < most; ++x) out[x] = s.at(x);
  return s.count;
}
int len_of(const int *lens, int slots, int cap, int slot) { return slot_len(lens, slots, cap, slot); }
int row_of(int page, int pages, int lp, int pos) { return page_row(page, pages, lp, pos); }
int chunk(long long total, int target, int step) { return chunk_len(total, target, step); }
int chunks(int count, int len) { return chunks_of(count, len); }
int chunk_stop(int x0, int count, int len) { return chunk_end(x0, count, len); }
int blocks(long long tokens, int lp) { return pages_of(tokens, lp); }
}
"""


@pytest.fixture(scope="module")
def idx(tmp_path_factory):
    d = tmp_path_factory.mktemp("idx")
    (d / "i.cpp").write_text(SRC)
    so = str(d / "i.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-std=c++17",
                    "-I", os.path.join(ROOT, "paper_2605_13433_amd", "csrc"), str(d / "i.cpp"),
                    "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.chunk.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    lib.blocks.argtypes = [ctypes.c_longlong, ctypes.c_int]
    return lib


def test_seen_tokens(idx):
    buf = (ctypes.c_int * 64)()
    for L in list(range(0, 9)) + [40]:
        for window in (0, 1, 2, 5, 8, 39, 40, 41, 2 ** 31 - 1):
            for sinks in (0, 1, 4, 9, 40, 2 ** 31 - 1):
                n = idx.seen_list(L, window, sinks, buf, 64)
                want = np.nonzero(seen(L, window, sinks)[L - 1])[0].tolist() if L else []
                assert list(buf[:n]) == want, (L, window, sinks)


def test_bad_slots_lengths_and_pages(idx):
    lens = (ctypes.c_int * 3)(5, -7, 1000)
    got = [idx.len_of(lens, 3, 64, s) for s in (-1, 0, 1, 2, 3, 2 ** 31 - 1, -2 ** 31)]
    assert got == [0, 5, 0, 64, 0, 0, 0]
    for lp in (0, 3, 10):
        P = 1 << lp
        pages = (2 ** 31 - 1) // P
        for page in (-2 ** 31, -1, pages, 2 ** 31 - 1):
            assert idx.row_of(page, pages, lp, 3) == -1
        for pos in (0, 1, P - 1, P, 12345678):
            assert idx.row_of(0, pages, lp, pos) == pos % P
            row = idx.row_of(pages - 1, pages, lp, pos)
            assert 0 <= row < pages * P and row == (pages - 1) * P + pos % P


@pytest.mark.parametrize("seed", range(30))
def test_chunks_fit_the_grid(idx, seed):
    """The chunks of all rows are at most target + rows, whatever the lengths."""
    rng = np.random.default_rng(seed)
    rows = int(rng.integers(1, 300))
    lens = np.exp(rng.uniform(0, np.log(131072), rows)).astype(np.int64) * \
        (rng.random(rows) < 0.9)
    target, step = int(rng.integers(1, 2000)), int(rng.choice([32, 64, 256]))
    C = idx.chunk(int(lens.sum()), target, step)
    assert C >= step and C % step == 0
    assert int(np.sum(-(-lens // C))) <= target + rows
    # the longest batch that the calls allow
    assert 0 < idx.chunk(65536 * 131072, 1024, 256) < 2 ** 31


@pytest.mark.parametrize("rows,count,target", [
    (65536, 2 ** 31 - 1, 1), (65536, 2 ** 31 - 1, 1024), (65536, 1 << 24, 16), (65536, 1 << 22, 128),
    (3, 2 ** 31 - 1, 1024), (2, 2 ** 30 + 1, 1), (1, 2 ** 31 - 1, 1), (1, 1, 1024), (65536, 1, 1)])
def test_chunks_of_the_longest_rows(idx, rows, count, target):
    """Many rows may name one long sequence: the chunks still fit the grid, follow each
    other and end with the row."""
    C = idx.chunk(rows * count, target, 256)
    n = idx.chunks(count, C)
    assert C > 0 and n == -(-count // C) and n * rows <= target + rows
    for x in {0, n // 2, n - 1}:
        assert idx.chunk_stop(x * C, count, C) == min((x + 1) * C, count)
    assert idx.chunks(0, C) == 0


def test_blocks(idx):
    for lp in (0, 4, 10):
        for n in (0, 1, (1 << lp) - 1, 1 << lp, (1 << lp) + 1, 2 ** 31 - 1):
            assert idx.blocks(n, lp) == -(-n // (1 << lp))


# ----------------------------------------------------------------------- model
@pytest.mark.parametrize("seed", range(6))
def test_model_keeps_every_history(seed):
    """Random calls: the invariants hold, and every sequence's tokens are what was
    written to it or to what it was forked from, wherever its pages went."""
    rng = np.random.default_rng(seed)
    P, pages, slots, cols = int(rng.choice([1, 4, 8])), 40, 7, 9
    k = rng.standard_normal((2, pages, P, 1))
    m = Model(k, k.copy(), np.zeros((pages, P), np.int64), slots, cols)
    want = [[] for _ in range(slots)]
    token = 0
    for _ in range(120):
        op = rng.integers(5)
        some = rng.integers(-1, slots + 1, rng.integers(1, slots + 1))
        if op <= 1:
            counts = rng.integers(-1, 3 * P, len(some))
            start = m.extend(some, counts)
            off = np.concatenate([[0], np.cumsum(np.maximum(counts, 0))])
            new = np.arange(token, token + off[-1], dtype=np.float64)
            token += int(off[-1])
            for layer in range(2):
                m.write(layer, new[:, None], -new[:, None], some, start, off, new.astype(np.int64))
            for r, s in enumerate(some):
                if start[r] >= 0:
                    assert start[r] == len(want[s])
                    want[s] = want[s] + list(new[off[r]:off[r + 1]])
        elif op == 2:
            src = rng.integers(0, slots, len(some))
            m.fork(src, some)
            old, seen_ = [list(x) for x in want], set()
            for s, d in zip(src, some):
                if 0 <= d < slots and d not in seen_:
                    want[d] = old[s]
                seen_.add(d)
        elif op == 3:
            m.free(some)
            for s in some:
                if 0 <= s < slots:
                    want[s] = []
        else:
            live = m.compact()
            assert (m.refs[:live] > 0).all() and (m.refs[live:] == 0).all()
        m.check()
        for s in range(slots):
            for layer in range(2):
                kk, vv, tt = m.history(s, layer)
                assert kk[:, 0].tolist() == want[s] and vv[:, 0].tolist() == [-x for x in want[s]]
                assert tt.tolist() == [int(x) for x in want[s]]


# -------------------------------------------------------------------- refusals
needs_lib = pytest.mark.skipif(not os.path.exists(hstu.LIB_PATH),
                               reason="libhstu_jagged.so not built")
FAKE = 0x1000   # never dereferenced


def _desc(**kw):
    f = dict(dtype=hstu.HSTU_BF16, layers=2, num_pages=10, page_size=16, H=4, d=64, slots=3,
             max_pages=5, k=FAKE, v=FAKE, ts=FAKE, tables=FAKE, lens=FAKE, refs=FAKE, status=FAKE)
    f.update(kw)
    return paged.CacheDesc(*[f[n] for n, _ in paged.CacheDesc._fields_])


def _calls(c):
    """Every call on the descriptor, with arguments that are right otherwise."""
    lib = paged._lib()
    c = ctypes.byref(c) if c is not None else None
    big = 1 << 40
    out = paged.PagedOut(FAKE, FAKE, FAKE, big)
    return {
        "clear": lambda: lib.hstu_cache_clear(c, None),
        "extend": lambda n=2, s=FAKE, ws=FAKE, b=big, start=FAKE: lib.hstu_cache_extend(
            c, s, FAKE, n, start, ws, b, None),
        "write": lambda layer=0, n=2, k=FAKE, ts=None, total=4, new=2: lib.hstu_cache_write(
            c, layer, k, FAKE, ts, FAKE, FAKE, FAKE, n, total, new, None),
        "fork": lambda n=2, dst=FAKE, ws=FAKE, b=big: lib.hstu_cache_fork(
            c, FAKE, dst, n, ws, b, None),
        "free": lambda n=2, s=FAKE: lib.hstu_cache_free(c, s, n, None),
        "compact": lambda live=FAKE, ws=FAKE, b=big: lib.hstu_cache_compact(c, live, ws, b, None),
        "paged": lambda layer=0, rows=2, N=64, rab=None, win=None, q=FAKE, out=out:
            lib.hstu_paged_attn_fwd(q, FAKE, c, layer, FAKE, rows, N, rab, win,
                                    ctypes.byref(out) if out is not None else None, None),
    }


@needs_lib
@pytest.mark.parametrize("kw,code,frag", [
    (dict(dtype=5), -1, "dtype"), (dict(layers=0), -1, "layers"),
    (dict(layers=20000), -2, "layers"), (dict(num_pages=0), -1, "num_pages"),
    (dict(page_size=0), -1, "page_size"), (dict(page_size=24), -1, "page_size"),
    (dict(page_size=2048), -1, "page_size"), (dict(H=0), -1, "H = 0"),
    (dict(H=65), -2, "H = 65"), (dict(d=48), -1, "d = 48"), (dict(d=32), -2, "bf16"),
    (dict(slots=0), -1, "slots"), (dict(slots=1 << 25), -2, "slots"),
    (dict(max_pages=0), -1, "max_pages"),
    (dict(num_pages=1 << 27), -2, "num_pages * page_size"),
    (dict(max_pages=1 << 27), -2, "max_pages * page_size"),
    (dict(k=None), -1, "non-null"), (dict(refs=None), -1, "non-null"),
    (dict(status=None), -1, "non-null"), (dict(v=FAKE + 8), -1, "16-byte"),
])
def test_bad_descriptors(kw, code, frag):
    c = _desc(**kw)
    for name, call in _calls(c).items():
        assert call() == code, name
        assert frag in hstu.last_error()
    lib = paged._lib()
    assert lib.hstu_cache_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.hstu_paged_attn_workspace_bytes(ctypes.byref(c), 2) == 0


@needs_lib
def test_null_descriptor():
    for call in _calls(None).values():
        assert call() == -1 and "NULL" in hstu.last_error()


@needs_lib
def test_bad_arguments():
    f = _calls(_desc())
    g = _calls(_desc(ts=None))
    rab_t = ctypes.byref(hstu.Rab(None, FAKE, None, 32))
    rab_a = ctypes.byref(hstu.Rab(FAKE, None, None, 0, float("nan")))
    small = paged.PagedOut(FAKE, FAKE, FAKE, 16)
    none = paged.PagedOut(FAKE, FAKE, None, 1 << 40)
    for call, code, frag in [
        (lambda: f["extend"](n=-1), -1, "n = -1"), (lambda: f["extend"](n=4), -1, "3 slots"),
        (lambda: f["extend"](s=None), -1, "non-null"),
        (lambda: f["extend"](start=None), -1, "non-null"),
        (lambda: f["extend"](ws=None), -3, "workspace"), (lambda: f["extend"](b=8), -3, "needed"),
        (lambda: f["extend"](ws=FAKE + 1), -1, "aligned"),
        (lambda: f["write"](layer=2), -1, "layer = 2"),
        (lambda: f["write"](layer=-1), -1, "layer = -1"),
        (lambda: f["write"](n=9), -1, "3 slots"), (lambda: f["write"](total=-1), -1, "total_rows"),
        (lambda: f["write"](new=-1), -1, "max_new"), (lambda: f["write"](k=None), -1, "non-null"),
        (lambda: f["write"](k=FAKE + 4), -1, "16-byte"),
        (lambda: g["write"](ts=FAKE), -1, "without ts"),
        (lambda: f["fork"](n=4), -1, "3 slots"), (lambda: f["fork"](dst=None), -1, "non-null"),
        (lambda: f["fork"](b=8), -3, "needed"), (lambda: f["free"](n=-2), -1, "n = -2"),
        (lambda: f["free"](s=None), -1, "non-null"),
        (lambda: f["compact"](live=None), -1, "non-null"),
        (lambda: f["compact"](ws=None), -3, "workspace"),
        (lambda: f["paged"](layer=2), -1, "layer = 2"), (lambda: f["paged"](rows=-1), -1, "rows"),
        (lambda: f["paged"](rows=70000), -2, "rows"), (lambda: f["paged"](N=0), -1, "max_len"),
        (lambda: f["paged"](N=70000), -2, "max_len"), (lambda: f["paged"](q=None), -1, "non-null"),
        (lambda: f["paged"](q=FAKE + 2), -1, "16-byte"),
        (lambda: f["paged"](out=None), -1, "out is NULL"),
        (lambda: f["paged"](rab=rab_a), -1, "alpha"),
        (lambda: g["paged"](rab=rab_t), -1, "without ts"),
        (lambda: f["paged"](win=ctypes.byref(hstu.Window(-1, 0))), -1, "window = -1"),
    ]:
        assert call() == code, frag
        assert frag in hstu.last_error(), (frag, hstu.last_error())


@needs_lib
def test_empty_calls():
    f = _calls(_desc())
    assert f["extend"](n=0) == 0 and f["fork"](n=0) == 0 and f["free"](n=0) == 0
    assert f["write"](n=0) == 0 and f["write"](total=0) == 0 and f["write"](new=0) == 0
    assert f["paged"](rows=0) == 0


@needs_lib
def test_python_refuses_before_it_allocates():
    with pytest.raises(hstu.HstuError, match="page_size"):
        paged.Cache(10, 24, 4, 64, 2, 4)
    with pytest.raises(ValueError, match="dtype"):
        import torch
        paged.Cache(10, 16, 4, 64, 2, 4, dtype=torch.float16)
