"""Windowed jagged attention (forward and backward) against the definition in
float64.

Tolerances, relative to the largest value of a tensor, as for the plain operator
(tests/gpu_util.py): 2e-2 in bf16 -- the operands a and dS, the output o and the
LayerNorm gradient dO are each rounded by 2^-8 of the value at most, and sums of
them stay a few such steps off -- and 1e-5 in fp32.  The tables' gradients have 1e-5
in bf16 too: q, k, v, dy are the same numbers on both sides, and what lies between
them and the tables (a, o, dO) is carried to 24 bits, as in fp32.
"""
import numpy as np
import pytest
import torch

from oracle import window as ref
from paper_2605_13433_amd import hstu, inputs
from tests.gpu_util import TOL, check, say, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def run(w, window, sinks, alpha=1.0, det=False, bwd=True):
    q, k, v, u, off = (to_dev(x) for x in (w.q, w.k, w.v, w.u, w.seq_offsets))
    pos, tw, ts = to_dev(w.pos_w), to_dev(w.time_w), to_dev(w.timestamps)
    plan = hstu.Plan(q, off, w.N, pos, tw, ts, w.num_buckets, backward=bwd, alpha=alpha,
                     deterministic=det, window=window, sinks=sinks)
    f = plan.forward(q, k, v, u, off)
    out = dict(o=f.o, y=f.y, mean=f.ln_mean, rstd=f.ln_rstd)
    if bwd:
        g = plan.backward(q, k, v, u, off, to_dev(w.dy))
        out.update(dq=g.dq, dk=g.dk, dv=g.dv, du=g.du, d_pos=g.d_pos_w, d_time=g.d_time_w)
    torch.cuda.synchronize()
    return out


def wide(t):
    return None if t is None else t.detach().to("cpu", torch.float64).numpy()


def against(w, window, sinks, alpha=1.0, det=False):
    say(f"  window {window} sinks {sinks} T {w.q.shape[0]} H {w.H} d {w.d} {w.q.dtype} "
        f"pos {w.pos_w is not None} time {w.time_w is not None}")
    got = run(w, window, sinks, alpha, det)
    f = lambda t: None if t is None else t.double().numpy()
    want = ref.attention(f(w.q), f(w.k), f(w.v), f(w.u), w.seq_offsets.numpy(), w.N, window, sinks,
                         f(w.pos_w), f(w.time_w), None if w.timestamps is None
                         else w.timestamps.numpy(), f(w.dy), alpha)
    tol = TOL[w.q.dtype]
    for n in ("o", "y", "dq", "dk", "dv", "du", "d_pos", "d_time"):
        if want[n] is not None:
            check(n, wide(got[n]), want[n].reshape(got[n].shape),
                  TOL[torch.float32] if n.startswith("d_") else tol)
    return got, want


LENS = [1, 70, 130, 0, 64, 65, 300, 63]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pos,time", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("window,sinks", [(64, 4), (1, 0), (50, 3)])
def test_bf16(d, pos, time, window, sinks):
    w = inputs.make_workload(LENS, H=2, d=d, N=320, pos=pos, time=time, seed=5 * d + window)
    against(w, window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (1, 64), (2, 65), (63, 0), (64, 0),
                                          (65, 1), (128, 130), (129, 63), (319, 0), (10, 200)])
@pytest.mark.parametrize("d", [64, 128])
def test_bf16_edges(d, window, sinks):
    w = inputs.make_workload(LENS, H=3, d=d, N=320, seed=window + 7 * sinks + d)
    against(w, window, sinks)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (1, 0), (31, 2), (32, 33), (33, 0),
                                          (100, 64), (65, 129)])
def test_f32(d, window, sinks):
    w = inputs.make_workload(LENS, H=2, d=d, N=320, dtype=torch.float32,
                             seed=window + 11 * sinks + d)
    against(w, window, sinks)


@pytest.mark.parametrize("window,sinks", [(17, 2), (64, 40)])
def test_f32_short_batches(window, sinks):
    # two waves an item: at most four tiles a sequence, more items than fit at once
    rng = np.random.default_rng(window)
    w = inputs.make_workload([int(x) for x in rng.integers(1, 129, 120)], H=8, d=64, N=128,
                             dtype=torch.float32, seed=window)
    against(w, window, sinks)


@pytest.mark.parametrize("window,sinks", [(40, 3), (64, 70), (200, 129), (0, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_far_sinks(d, window, sinks):
    # several chunks of query tiles behind the sinks' windows, one and two heads' worth
    w = inputs.make_workload([1500, 2300, 900, 64, 4000], H=1, d=d, N=4000,
                             seed=window + sinks + d)
    against(w, window, sinks)


@pytest.mark.parametrize("pos,time", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("d", [64, 128])
def test_far_sinks_and_tables(d, pos, time):
    w = inputs.make_workload([3000, 70, 1], H=2, d=d, N=3000, pos=pos, time=time, seed=77)
    against(w, 100, 66)


@pytest.mark.parametrize("d", [64, 128])
def test_far_sinks_among_many_items(d):
    # long chains in a batch whose backward takes two launches
    rng = np.random.default_rng(d)
    lens = [int(x) for x in rng.integers(0, 400, 350)] + [4000, 2500]
    w = inputs.make_workload(lens, H=2, d=d, N=4000, seed=78)
    against(w, 60, 70)


@pytest.mark.parametrize("d,H,n,window,sinks", [(64, 4, 400, 100, 5), (128, 2, 250, 90, 0),
                                                (64, 2, 700, 30, 66)])
def test_many_items(d, H, n, window, sinks):
    # more items than run at once: the persistent kernels, each backward in two launches
    rng = np.random.default_rng(n)
    w = inputs.make_workload([int(x) for x in rng.integers(0, 400, n)], H=H, d=d, N=400, seed=n)
    against(w, window, sinks)


def test_pairs_of_query_tiles():
    # mean length above 256 at d = 64: items of two query tiles
    rng = np.random.default_rng(1)
    w = inputs.make_workload([int(x) for x in rng.integers(200, 700, 60)], H=2, d=64, N=700, seed=9)
    against(w, 77, 9)


@pytest.mark.parametrize("alpha", [0.125, -1.5])
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128),
                                     (torch.float32, 64)])
def test_alpha(dtype, d, alpha):
    w = inputs.make_workload([90, 5, 200], H=2, d=d, N=200, dtype=dtype, seed=21)
    against(w, 70, 2, alpha=alpha)


@pytest.mark.parametrize("d", [64, 128])
def test_deterministic_repeats(d):
    w = inputs.make_workload([900, 300, 77, 1500], H=2, d=d, N=1500, seed=31)
    a, _ = against(w, 150, 40, det=True)
    b = run(w, 150, 40, det=True)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128),
                                     (torch.float32, 32)])
def test_wide_window_is_the_plain_operator(dtype, d):
    w = inputs.make_workload([300, 1, 129, 0, 512], H=2, d=d, N=512, dtype=dtype, seed=41)
    plain = run(w, None, 0)
    for window, sinks in ((512, 0), (0, 512), (1 << 30, 1 << 30)):
        got = run(w, window, sinks)
        for n in plain:
            check(n, wide(got[n]), wide(plain[n]), TOL[dtype])


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128),
                                     (torch.float32, 64)])
def test_empty_rows(dtype, d):
    """window 0: only the sinks are seen, and with none of those nothing is."""
    w = inputs.make_workload([100, 64, 3], H=2, d=d, N=100, dtype=dtype, seed=51)
    got = run(w, 0, 0)
    for n in ("o", "y", "dq", "dk", "dv", "du", "d_pos", "d_time"):
        assert torch.count_nonzero(got[n]) == 0, n


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128),
                                     (torch.float32, 64)])
def test_unseen_rows_leave_no_trace(dtype, d, bad):
    """Rows of k and v that hold no numbers reach the rows that see them alone, and a
    row of dy the rows that its own row sees."""
    window, sinks, L = 50, 3, 400
    w = inputs.make_workload([30, L, 40], H=2, d=d, N=L, dtype=dtype, seed=61)
    clean = {n: wide(t) for n, t in run(w, window, sinks).items()}
    at, row = 30, 170
    m = ref.seen(L, window, sinks)
    # k and v of one token
    w.k[at + row, 1, 5] = bad
    w.v[at + row, 0, 7] = bad
    got = {n: wide(t) for n, t in run(w, window, sinks).items()}
    hit = np.zeros(w.q.shape[0], bool)
    hit[at:at + L] = m[:, row]
    for n in ("o", "y"):
        check(n, got[n][~hit], clean[n][~hit], TOL[dtype])
        assert not np.isfinite(got[n][hit]).all(axis=tuple(range(1, got[n].ndim))).any(), n
    touched = np.zeros(w.q.shape[0], bool)           # rows that some hit row sees
    touched[at:at + L] = m[hit[at:at + L]].any(0)
    for n in ("dq", "du"):
        check(n, got[n][~hit], clean[n][~hit], TOL[dtype])
    for n in ("dk", "dv"):
        check(n, got[n][~touched], clean[n][~touched], TOL[dtype])
    # q and dy of one token
    w = inputs.make_workload([30, L, 40], H=2, d=d, N=L, dtype=dtype, seed=61)
    w.q[at + row, 1, 5] = bad
    w.dy.view(len(w.dy), -1)[at + row, 9] = bad
    got = {n: wide(t) for n, t in run(w, window, sinks).items()}
    own = np.zeros(w.q.shape[0], bool)
    own[at + row] = True
    for n in ("o", "y", "dq", "du"):
        check(n, got[n][~own], clean[n][~own], TOL[dtype])
    touched[:] = False
    touched[at:at + L] = m[row]
    for n in ("dk", "dv"):
        check(n, got[n][~touched], clean[n][~touched], TOL[dtype])


@pytest.mark.parametrize("pos,time", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("L", [50, 64, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_unseen_rows_of_the_first_tile(d, L, pos, time):
    """As above for a row of the first tile, with and without tables (which sum dQ of
    those rows in different places); the rows before it must not see it."""
    w = inputs.make_workload([L, 3, L], H=2, d=d, N=L, pos=pos, time=time, seed=62)
    row, window, sinks = 40, 30, 2
    clean = {n: wide(t) for n, t in run(w, window, sinks).items() if t is not None}
    w.k[L + 3 + row, 0, 1] = float("nan")
    w.v[L + 3 + row, 1, 1] = float("inf")
    got = {n: wide(t) for n, t in run(w, window, sinks).items() if t is not None}
    m = ref.seen(L, window, sinks)
    hit = np.zeros(2 * L + 3, bool)
    hit[L + 3:] = m[:, row]
    for n in ("o", "y", "dq", "du"):
        check(n, got[n][~hit], clean[n][~hit], TOL[torch.bfloat16])


def test_differences():
    """The gradients in fp32 along random directions against central differences of
    the forward in float64 (the definition)."""
    w = inputs.make_workload([40, 90], H=2, d=32, N=90, dtype=torch.float32, seed=71)
    got = run(w, 20, 2)
    f = lambda t: t.double().numpy()
    base = dict(q=f(w.q), k=f(w.k), v=f(w.v), u=f(w.u), pos_w=f(w.pos_w), time_w=f(w.time_w))
    rng = np.random.default_rng(0)

    def loss(x):
        r = ref.attention(x["q"], x["k"], x["v"], x["u"], w.seq_offsets.numpy(), w.N, 20, 2,
                          x["pos_w"], x["time_w"], w.timestamps.numpy())
        return float((r["y"] * f(w.dy).reshape(r["y"].shape)).sum())

    for name, g in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("u", "du"), ("pos_w", "d_pos"),
                    ("time_w", "d_time")):
        step = rng.standard_normal(base[name].shape)
        eps = 1e-5
        up, down = ({**base, name: base[name] + s * eps * step} for s in (1, -1))
        want = (loss(up) - loss(down)) / (2 * eps)
        have = float((wide(got[g]).reshape(step.shape) * step).sum())
        # the differences' own error (third derivatives) is of the order eps^2; the
        # gradient's is 1e-5 of its largest value for each of its entries
        scale = float(np.abs(wide(got[g])).max()) * np.abs(step).sum() * 1e-5 + 1e-7 * abs(want)
        say(f"    {name}: {have:.9g} against {want:.9g} (bound {scale:.2g})")
        assert abs(have - want) <= scale


def test_two_streams_and_a_graph():
    w = inputs.make_workload([300, 90, 700], H=2, d=64, N=700, seed=81)
    q, k, v, u, off, dy = (to_dev(x) for x in (w.q, w.k, w.v, w.u, w.seq_offsets, w.dy))
    pos, tw, ts = to_dev(w.pos_w), to_dev(w.time_w), to_dev(w.timestamps)

    def plan():
        return hstu.Plan(q, off, w.N, pos, tw, ts, w.num_buckets, window=100, sinks=5,
                         deterministic=True)

    def outs(f, g):
        return [t.clone() for t in (f.y, f.o, g.dq, g.dk, g.dv, g.du, g.d_pos_w, g.d_time_w)]

    p0 = plan()
    want = outs(p0.forward(q, k, v, u, off), p0.backward(q, k, v, u, off, dy))
    torch.cuda.synchronize()
    # side by side on two streams, each with its own plan
    plans, streams = [plan(), plan()], [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for p, s in zip(plans, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(outs(p.forward(q, k, v, u, off), p.backward(q, k, v, u, off, dy)))
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g, want):
            assert torch.equal(a, b)
    # captured and replayed, eager work in between
    p = plan()
    p.forward(q, k, v, u, off), p.backward(q, k, v, u, off, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f, g = p.forward(q, k, v, u, off), p.backward(q, k, v, u, off, dy)
    for _ in range(4):
        for t in (f.y, f.o, g.dq, g.dk, g.dv, g.du, g.d_pos_w, g.d_time_w):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs(f, g), want):
            assert torch.equal(a, b)
        p0.forward(q, k, v, u, off)


@pytest.mark.parametrize("window,sinks", [(40, 0), (0, 3), (64, 70)])
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128),
                                     (torch.float32, 32)])
def test_batches_without_tokens(dtype, d, window, sinks):
    for lens in ([], [0], [0, 0, 0]):
        w = inputs.make_workload(lens, H=2, d=d, N=100, dtype=dtype, seed=71)
        got = run(w, window, sinks)
        assert got["dq"].shape[0] == 0 and got["y"].shape[0] == 0
        for n in ("d_pos", "d_time"):
            assert torch.count_nonzero(got[n]) == 0, n


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128),
                                     (torch.float32, 64)])
def test_checked_offsets(monkeypatch, dtype, d):
    """HSTU_VALIDATE=1: valid offsets give what an unchecked call gives, others are
    reported and no pair is worked on."""
    w = inputs.make_workload([300, 0, 1, 129], H=2, d=d, N=300, dtype=dtype, seed=73)
    plain = run(w, 70, 5, det=True)
    monkeypatch.setenv("HSTU_VALIDATE", "1")
    q, k, v, u, off = (to_dev(x) for x in (w.q, w.k, w.v, w.u, w.seq_offsets))
    plan = hstu.Plan(q, off, w.N, to_dev(w.pos_w), to_dev(w.time_w), to_dev(w.timestamps),
                     w.num_buckets, backward=True, deterministic=True, window=70, sinks=5)
    f = plan.forward(q, k, v, u, off)
    assert plan.status() == 0
    g = plan.backward(q, k, v, u, off, to_dev(w.dy))
    assert plan.status(backward=True) == 0
    for n, t in (("y", f.y), ("dq", g.dq), ("dk", g.dk), ("dv", g.dv), ("d_pos", g.d_pos_w),
                 ("d_time", g.d_time_w)):
        check(n, wide(t), wide(plain[n]), TOL[torch.float32] if n.startswith("d_") else TOL[dtype])
    bad = off.clone()
    bad[1], bad[2] = 310, 300                              # too long, then decreasing
    bits = hstu.HSTU_SEQ_TOO_LONG | hstu.HSTU_SEQ_DECREASING
    plan.forward(q, k, v, u, bad)
    assert plan.status() == bits
    g = plan.backward(q, k, v, u, bad, to_dev(w.dy))
    assert plan.status(backward=True) == bits
    assert torch.isfinite(g.d_pos_w).all() and torch.isfinite(g.d_time_w).all()


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("B,N,window,sinks", [(256, 2048, 64, 4), (40, 4096, 500, 130), (3, 300, 9, 1)])
def test_a_workspace_holds_for_fewer_tokens(B, N, window, sinks, bias):
    t = torch.zeros(1, device="cuda")
    rab = hstu.make_rab(t if bias else None, None, None, 128, 1.0)
    win = hstu.make_window(window, sinks, t)
    sizes = [hstu.hstu_jagged_window_attn_workspace_bytes(B, N, 4, 64, T, 1, hstu.HSTU_BF16, rab, win)
             for T in sorted((1, 100, 1000, 5000, 20000, 60000, B * N // 2, B * N))]
    assert sizes == sorted(sizes)
