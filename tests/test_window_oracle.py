"""The float64 windowed attention (oracle/window.py) against what does not share its
formulas: the plain operator's oracle, torch's autograd over a dense form, the
pair rule counted by hand."""
import os

import numpy as np
import pytest
import torch

from oracle import window as ref
from paper_2605_13433_amd import inputs

GOLDEN = os.path.join(os.path.dirname(__file__), "golden", "time_buckets.txt")


def _f(t):
    return None if t is None else t.double().numpy()


def _run(w, window, sinks, alpha=1.0):
    return ref.attention(_f(w.q), _f(w.k), _f(w.v), _f(w.u), w.seq_offsets.numpy(), w.N, window,
                         sinks, _f(w.pos_w), _f(w.time_w), w.timestamps.numpy(), _f(w.dy), alpha)


def test_pairs_by_hand():
    want = {(0, 0): [], (0, 1): [0], (1, 0): [4], (2, 0): [3, 4], (2, 1): [0, 3, 4],
            (2, 3): [0, 1, 2, 3, 4], (9, 0): [0, 1, 2, 3, 4], (0, 9): [0, 1, 2, 3, 4]}
    for (window, sinks), cols in want.items():
        assert np.nonzero(ref.seen(5, window, sinks)[4])[0].tolist() == cols


def test_whole_window_is_the_plain_operator(oracle_lib):
    w = inputs.make_workload([5, 70, 0, 33], H=2, d=64, N=80, seed=3)
    got = _run(w, 80, 0)
    want = dict(oracle_lib.fwd_workload(w), **oracle_lib.bwd_workload(w))
    for n, x in got.items():
        assert np.allclose(x.ravel(), want[n].ravel(), atol=1e-12, rtol=0), n


def test_buckets():
    lines = [x.split() for x in open(GOLDEN)
             if x.strip() and not x.startswith("#")]
    for x, b in lines:
        assert ref.bucket(int(x), 128) == int(b)


@pytest.mark.parametrize("window,sinks,alpha", [(0, 2, 1.0), (1, 0, 1.0), (7, 3, 0.5), (20, 0, 1.0)])
def test_gradients_against_autograd(window, sinks, alpha):
    w = inputs.make_workload([1, 23, 0, 12], H=2, d=32, N=30, dtype=torch.float32, seed=window)
    T, H, d = w.q.shape
    leaf = {n: t.double().clone().requires_grad_() for n, t in
            dict(q=w.q, k=w.k, v=w.v, u=w.u.view(T, H * d), pos=w.pos_w, time=w.time_w).items()}
    rows = []
    off = w.seq_offsets.tolist()
    for b in range(w.B):
        r = slice(off[b], off[b + 1])
        L = r.stop - r.start
        if L == 0:
            continue
        i, j = torch.arange(L)[:, None], torch.arange(L)[None, :]
        t = w.timestamps[r]
        bk = torch.tensor(ref.bucket((t[:, None] - t[None, :]).numpy(), w.time_w.shape[1]))
        s = alpha * torch.einsum("ihc,jhc->hij", leaf["q"][r], leaf["k"][r]) \
            + leaf["pos"][:, (j - i + w.N - 1).expand(L, L)] + leaf["time"][:, bk]
        m = (i >= j) & ((j > i - window) | (sinks > j))
        a = torch.nn.functional.silu(s) * m / w.N
        rows.append(torch.einsum("hij,jhc->ihc", a, leaf["v"][r]).reshape(L, H * d))
    y = torch.nn.functional.layer_norm(torch.cat(rows), (H * d,), eps=1e-6) * leaf["u"]
    (y * w.dy.double().view(T, H * d)).sum().backward()
    got = _run(w, window, sinks, alpha)
    assert np.allclose(got["y"], y.detach().numpy(), atol=1e-11)
    for n, g in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("u", "du"), ("pos", "d_pos"),
                 ("time", "d_time")):
        want = leaf[n].grad.numpy()
        assert np.allclose(got[g], want, atol=1e-9 * max(1.0, np.abs(want).max())), n


def test_one_token_is_the_last_row():
    w = inputs.make_workload([41], H=2, d=32, N=50, dtype=torch.float32, seed=4)
    for window, sinks in ((50, 0), (7, 3), (0, 2), (0, 0), (1, 0)):
        full = ref.attention(_f(w.q), _f(w.k), _f(w.v), _f(w.u), w.seq_offsets.numpy(), w.N,
                             window, sinks, _f(w.pos_w), _f(w.time_w), w.timestamps.numpy())
        o, y = ref.one_token(_f(w.q)[-1], _f(w.u)[-1].ravel(), _f(w.k), _f(w.v), w.N, window,
                             sinks, _f(w.pos_w), _f(w.time_w), w.timestamps.numpy())
        assert np.allclose(o, full["o"][-1], atol=1e-13)
        assert np.allclose(y, full["y"][-1], atol=1e-12)
