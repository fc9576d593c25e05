"""Host-side argument checks of the windowed attention (no GPU needed: every case
is rejected, or empty, before the library touches a device)."""
import ctypes
import os

import pytest

from paper_2605_13433_amd import hstu

pytestmark = pytest.mark.skipif(not os.path.exists(hstu.LIB_PATH),
                                reason="libhstu_jagged.so not built")

FAKE = 0x1000   # never dereferenced


def _win(window, sinks):
    return ctypes.byref(hstu.Window(window, sinks))


def _fwd(win, T=10, q=FAKE, d=64, dtype=hstu.HSTU_BF16):
    out = hstu.FwdOut(dtype, T, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30)
    return hstu.load_library().hstu_jagged_window_attn_fwd(
        q, FAKE, FAKE, FAKE, FAKE, 2, 64, 2, d, None, win, ctypes.byref(out), None)


def _bwd(win, T=10, dq=FAKE, rab=None):
    io = hstu.BwdIO(hstu.HSTU_BF16, T, FAKE, FAKE, FAKE, FAKE, dq, FAKE, FAKE, FAKE, None, None,
                    FAKE, 1 << 30)
    return hstu.load_library().hstu_jagged_window_attn_bwd(
        FAKE, FAKE, FAKE, FAKE, FAKE, 2, 64, 2, 64, ctypes.byref(rab) if rab else None, win,
        ctypes.byref(io), None)


@pytest.mark.parametrize("win,frag", [(None, "win is NULL"), ((-1, 0), "window = -1"),
                                      ((4, -2), "sinks = -2")])
def test_bad_windows(win, frag):
    w = None if win is None else _win(*win)
    for call in (_fwd, _bwd):
        assert call(w) == -1
        assert frag in hstu.last_error()
    assert hstu.load_library().hstu_jagged_window_attn_workspace_bytes(
        2, 64, 2, 64, 10, 1, hstu.HSTU_BF16, None, w) == 0
    assert frag in hstu.last_error()


def test_the_plain_checks_hold():
    assert _fwd(_win(4, 0), q=None) == -1 and "non-null" in hstu.last_error()
    assert _fwd(_win(4, 0), d=48) == -1 and "d = 48" in hstu.last_error()
    assert _fwd(_win(4, 0), d=32) == -2
    assert _fwd(_win(4, 0), dtype=9) == -1 and "dtype" in hstu.last_error()
    assert _bwd(_win(4, 0), dq=None) == -1 and "dq" in hstu.last_error()
    assert _bwd(_win(4, 0), rab=hstu.Rab(FAKE, None, None, 0)) == -1
    assert "d_pos_w" in hstu.last_error()


def test_the_tables_need_o():
    io = hstu.BwdIO(hstu.HSTU_BF16, 10, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None,
                    FAKE, 1 << 40)
    rab = hstu.Rab(FAKE, None, None, 0)
    rc = hstu.load_library().hstu_jagged_window_attn_bwd(
        FAKE, FAKE, FAKE, FAKE, FAKE, 2, 64, 2, 64, ctypes.byref(rab), _win(4, 0),
        ctypes.byref(io), None)
    assert rc == -1 and "o_full" in hstu.last_error()


def test_empty_batches():
    assert _fwd(_win(0, 0), T=0) == 0
    assert _bwd(_win(0, 0), T=0) == 0


def test_python_refusals():
    with pytest.raises(ValueError, match="without a window"):
        hstu.make_window(None, 3)
    assert hstu.make_window(None) is None
    for window, sinks in ((-1, 0), (1 << 31, 0), ((1 << 32) + 5, 0), (5, -1), (5, 1 << 32)):
        with pytest.raises(ValueError, match="not in"):
            hstu.make_window(window, sinks)
    w = hstu.make_window((1 << 31) - 1, 0)
    assert (w.window, w.sinks) == ((1 << 31) - 1, 0)
