"""Oracle of the gated linear recurrence against differences and identities, and the refusals of its entry points and
binding (CPU only: fake aligned addresses stand in for device buffers, nothing is dereferenced)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import recur as OR
from tests.test_history_cpu import A, central, close, hg, rows, seq  # noqa: F401

FAR = [(k + 2) << 34 for k in range(12)]  # arrays that share nothing, whatever their sizes here


@pytest.mark.parametrize("lens", [None, [0, 1, 4], [4, 3, 2]])
@pytest.mark.parametrize("state", [False, True])
def test_gradients(lens, state):
    rng = np.random.default_rng(3)
    n, T, d = 3, 4, 2
    x, g, dy = rng.standard_normal((3, n, T, d))
    bias = rng.standard_normal(d)
    h, dh = rng.standard_normal((2, n, d)) if state else (np.zeros((n, d)), np.zeros((n, d)))
    lens = None if lens is None else np.array(lens)

    def both():
        y, last, _, _ = OR.forward(x, g, bias, lens, h)
        return np.concatenate([y.ravel(), last.ravel()])

    up = np.concatenate([dy.ravel(), dh.ravel()])
    got, mag = OR.backward(x, g, dy, bias, lens, h, dh)
    for v, k in ((x, "dx"), (g, "dg"), (bias, "dbias"), (h, "dh_in")):
        close(got[k], central(both, v, up))
        assert (np.abs(got[k]) <= mag[k] + 1e-12).all()


def test_recurrence_is_the_weighted_sum_and_splits():
    rng = np.random.default_rng(4)
    T, d = 9, 5
    x, g = rng.standard_normal((2, 1, T, d))
    z = 1 / (1 + np.exp(-g[0]))
    want = sum(np.prod(1 - z[u + 1:], 0) * z[u] * x[0, u] for u in range(T))
    y, h, _, _ = OR.forward(x, g)
    close(h[0], want, 1e-12)
    _, a, _, _ = OR.forward(x[:, :4], g[:, :4])
    y2, b, _, _ = OR.forward(x[:, 4:], g[:, 4:], None, None, a)
    close(b, h, 1e-12)
    close(y2, y[:, 4:], 1e-12)


def params(hg, d=128, dt=1, bias=None):  # noqa: F811
    return ctypes.byref(hg.hg_recur_params(d, dt, bias))


def test_sizes(hg):  # noqa: F811
    so = hg.lib()
    s, w = ctypes.c_size_t(), ctypes.c_size_t()

    def query(n=3, T=40, **k):
        return so.hg_recur_workspace_size(params(hg, **k), n, T, ctypes.byref(s), ctypes.byref(w))

    assert query() == 0 and s.value == 4 * 3 * 2 * 128 and w.value >= 4 * 128  # two of every sixteen states
    assert query(T=16) == 0 and s.value == 0
    assert query(T=17) == 0 and s.value == 4 * 3 * 128
    assert query(n=0) == query(T=0) == 0 and s.value == 0
    assert query(n=1 << 20, T=1 << 26, d=16384) == 0 and s.value == 4 * (1 << 20) * ((1 << 22) - 1) * 16384
    for d in (0, 4, 12, -8, 16392):
        assert query(d=d) == 2
    assert query(dt=2) == query(dt=-1) == 2
    assert query(n=-1) == query(T=-1) == query(n=1 << 28) == query(T=1 << 30) == query(n=1 << 20, T=1 << 27) == 1
    assert query(bias=A + 8) == 1
    assert so.hg_recur_workspace_size(None, 1, 1, ctypes.byref(s), ctypes.byref(w)) == 1
    assert so.hg_recur_workspace_size(params(hg), 1, 1, None, ctypes.byref(w)) == 1
    assert so.hg_recur_workspace_size(params(hg), 1, 1, ctypes.byref(s), None) == 1


def test_forward_refusals(hg):  # noqa: F811
    so = hg.lib()
    null = ctypes.POINTER(hg.hg_seq)()

    def fwd(x=None, g=None, y=None, n=3, T=5, lens=None, h_in=FAR[3], h_out=FAR[4], saved=FAR[5], **k):
        r = [seq(hg, p) if v is None else v for v, p in ((x, FAR[0]), (g, FAR[1]), (y, FAR[2]))]
        return so.hg_recur_fwd(params(hg, **k), r[0], r[1], lens, n, T, h_in, r[2], h_out, saved, None)

    assert fwd(n=-1) == fwd(T=-1) == 1 and fwd(d=20) == fwd(dt=3) == 2
    assert fwd(x=null) == fwd(g=null) == fwd(y=null) == 1
    assert fwd(n=0, x=null) == 0
    assert fwd(x=seq(hg, A + 4)) == fwd(g=seq(hg, A, st=-128)) == fwd(x=seq(hg, A, sn=4100)) == 1
    assert fwd(y=seq(hg, FAR[2], st=64)) == fwd(y=seq(hg, FAR[2], sn=512)) == fwd(y=seq(hg, FAR[2], sn=0)) == 1
    assert fwd(h_in=A + 4) == fwd(h_out=A + 8) == fwd(saved=A + 128) == fwd(bias=A + 2) == 1
    row = 3 * 128 * 4
    # an output in another array's place, or part of it
    assert fwd(y=seq(hg, FAR[0])) == fwd(y=seq(hg, FAR[1] + 256)) == fwd(h_out=FAR[3] + 16) == fwd(h_out=FAR[0] + 256) == 1
    assert fwd(h_out=FAR[2]) == fwd(h_in=FAR[2] + 256) == fwd(h_in=FAR[2] + 8192 - row + 16) == 1
    assert fwd(T=40, saved=FAR[0]) == fwd(T=40, saved=FAR[3]) == fwd(T=40, saved=FAR[2]) == fwd(T=40, saved=FAR[4]) == 1
    assert fwd(y=seq(hg, A), bias=A) == fwd(h_out=A, bias=A + 16) == fwd(h_out=A, lens=A) == 1


def test_backward_refusals(hg):  # noqa: F811
    so = hg.lib()
    null = ctypes.POINTER(hg.hg_seq)()
    names = ("x", "g", "dy", "dx", "dg")

    def bwd(n=3, T=40, h_in=FAR[5], saved=FAR[6], dh_out=FAR[7], dh_in=FAR[8], db=FAR[9], scratch=FAR[10], lens=None,
            **k):
        r = [k.pop(v, seq(hg, FAR[i], 1 << 20)) for i, v in enumerate(names)]
        return so.hg_recur_bwd(params(hg, **k), r[0], r[1], lens, n, T, h_in, saved, r[2], dh_out, r[3], r[4], dh_in,
                               db, scratch, None)

    assert bwd(n=-1) == bwd(T=-1) == 1 and bwd(d=20) == 2
    for v in names:
        assert bwd(**{v: null}) == bwd(**{v: seq(hg, A + 8)}) == 1
    assert bwd(dx=seq(hg, FAR[3], 0)) == bwd(dg=seq(hg, FAR[4], st=64)) == 1
    assert bwd(saved=None) == bwd(saved=A + 16) == bwd(scratch=None) == bwd(scratch=A + 16) == 1
    assert bwd(dh_in=A + 4) == bwd(dh_out=A + 4) == bwd(h_in=A + 4) == 1
    s = lambda i, off=0: seq(hg, FAR[i] + off, 1 << 20)  # noqa: E731
    assert bwd(dx=s(0)) == bwd(dx=s(1)) == bwd(dx=s(2)) == bwd(dx=s(4)) == bwd(dg=s(0, 256)) == bwd(dg=s(2)) == 1
    assert bwd(dx=s(5)) == bwd(dg=s(6)) == bwd(dx=s(7)) == bwd(dg=s(8)) == bwd(dx=s(9)) == bwd(dg=s(10)) == 1
    assert bwd(dh_in=FAR[5]) == bwd(dh_in=FAR[7] + 16) == bwd(dh_in=FAR[6]) == bwd(dh_in=FAR[0]) == 1
    assert bwd(db=FAR[0]) == bwd(db=FAR[5]) == bwd(db=FAR[6]) == bwd(db=FAR[10]) == bwd(db=FAR[8]) == 1
    assert bwd(scratch=FAR[1]) == bwd(scratch=FAR[7]) == bwd(scratch=FAR[5]) == bwd(bias=FAR[9]) == 1


def test_step_refusals(hg):  # noqa: F811
    so = hg.lib()
    null = ctypes.POINTER(hg.hg_rows)()

    def step(x=None, g=None, y=None, n=10, live=None, h_in=FAR[3], h_out=FAR[4], **k):
        r = [rows(hg, p) if v is None else v for v, p in ((x, FAR[0]), (g, FAR[1]), (y, FAR[2]))]
        return so.hg_recur_step(params(hg, **k), r[0], r[1], live, n, h_in, r[2], h_out, None)

    assert step(n=-1) == 1 and step(d=20) == 2 and step(n=0, x=null) == 0
    assert step(x=null) == step(g=null) == step(y=null) == step(h_in=None) == step(h_out=None) == 1
    assert step(x=rows(hg, A + 2)) == step(g=rows(hg, A, 132)) == step(y=rows(hg, FAR[2], 64)) == 1
    assert step(h_in=A + 4) == step(h_out=A + 8) == step(h_out=FAR[3] + 64) == 1
    assert step(y=rows(hg, FAR[0])) == step(y=rows(hg, FAR[1] + 128)) == step(y=rows(hg, FAR[3])) == 1
    assert step(h_out=FAR[0]) == step(h_out=FAR[2]) == step(h_out=A, bias=A) == step(h_out=A, live=A) == 1


def test_a_large_array_between_the_sequences_of_another(hg):  # noqa: F811
    """The overlap check answers at once where a long array lies in the gaps of another.  (What it is asked to refuse is
    the last thing it looks at: lens within `saved`.)"""
    import time
    so = hg.lib()
    gap, n, T = 1 << 33, 4, 1 << 20  # values between two sequences of rows of 128 bf16 values
    saved = FAR[0] + 4 * T * 256     # 4 * 65535 * 512 bytes, in the gap
    t = time.perf_counter()
    assert so.hg_recur_fwd(params(hg), seq(hg, FAR[0], gap, 128), seq(hg, FAR[0] + T * 256, gap, 128), saved + 4096, n, T,
                           None, seq(hg, FAR[0] + 2 * T * 256, gap, 128), None, saved, None) == 1
    assert b"saved must not overlap" in so.hg_last_error()
    assert time.perf_counter() - t < 0.1


def test_binding_refuses_what_it_would_read_wrongly(hg):  # noqa: F811
    with pytest.raises(ValueError, match="storage types"):
        hg.RecurParams(d=8, dtype=torch.float16)
    with pytest.raises(ValueError, match="device memory"):
        hg.RecurParams(torch.zeros(8))
    p = hg.RecurParams(d=8, dtype=torch.float32)
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="device memory"):
        hg.hg_recur_fwd(p, x, x, None, None, x, None, None)
    with pytest.raises(ValueError, match="shape"):
        hg.hg_recur_fwd(p, x[..., :4], x, None, None, x, None, None)
    with pytest.raises(ValueError, match="shape"):
        hg.hg_recur_step(p, x[:, 0].double(), x[:, 0], None, x[:, 0], x[:, 0])


@pytest.mark.parametrize("dt", [0, 1])
def test_sizes_serve_smaller_calls(hg, dt):  # noqa: F811
    """What is enough for n sequences of up to T positions is enough for fewer or shorter ones."""
    so = hg.lib()
    s, w = ctypes.c_size_t(), ctypes.c_size_t()

    def query(n, T, d):
        assert so.hg_recur_workspace_size(params(hg, d, dt), n, T, ctypes.byref(s), ctypes.byref(w)) == 0
        return s.value, w.value

    Ts = [0, 1, 2, 12, 16, 17, 40, 64, 65, 300, 515, 1001, 4096, 32768, 1 << 20]
    ns = [1, 2, 3, 7, 40, 77, 400, 1000, 2000, 2700, 3000, 5000, 20000, 150001, 1 << 21]
    for d in (8, 64, 128, 264, 1024, 16384):
        grid = {(n, T): query(n, T, d) for n in ns for T in Ts}
        for i, n in enumerate(ns):
            for j, T in enumerate(Ts):
                here = grid[n, T]
                for less in ([(ns[i - 1], T)] if i else []) + ([(n, Ts[j - 1])] if j else []):
                    assert all(a >= b for a, b in zip(here, grid[less])), (d, n, T, less)


def test_sizes_asked_for_by_several_threads(hg):  # noqa: F811
    """Sizes of more shapes than are kept, of parameters that threads share: one that another thread drops between its
    asking and its return is still returned."""
    p = hg.RecurParams(d=8, dtype=torch.float32)

    class Dropping(dict):
        def __setitem__(self, key, value):
            dict.__setitem__(self, key, value)
            self.clear()  # as the other thread would

    p.__dict__["_known"] = Dropping()
    want = [(0, hg.hg_recur_workspace_size(hg.RecurParams(d=8, dtype=torch.float32), n, 3)[1]) for n in (1, 5, 900)]
    assert [hg.hg_recur_workspace_size(p, n, 3) for n in (1, 5, 900)] == want
