"""Oracle of the layer of experts against identities, and the refusals of its entry points and binding (CPU only: fake
aligned addresses stand in for device buffers, nothing is dereferenced)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import history as OH
from oracle import moe as OM
from tests.test_history_cpu import A, close, hg  # noqa: F401

FAR = [(k + 2) << 36 for k in range(12)]  # arrays that share nothing


def test_one_expert_is_the_block():
    rng = np.random.default_rng(0)
    X, Wr = rng.standard_normal((5, 6)), rng.standard_normal((6, 1))
    Wg, Wu = rng.standard_normal((2, 1, 6, 8))
    Wd = rng.standard_normal((1, 8, 6))
    for res in (False, True):
        Y, idx, w, _, _ = OM.forward(X, Wr, Wg, Wu, Wd, 1, "silu", res, False)
        close(Y, OH.ffn_forward(X, Wg[0], Wu[0], Wd[0], "silu", res), 1e-12)
        assert (idx == 0).all() and (w == 1).all()


def test_all_experts_are_the_weighted_sum_and_ties_go_down():
    rng = np.random.default_rng(1)
    X, Wr = rng.standard_normal((5, 6)), rng.standard_normal((6, 4))
    Wg, Wu = rng.standard_normal((2, 4, 6, 8))
    Wd = rng.standard_normal((4, 8, 6))
    Y, idx, w, _, _ = OM.forward(X, Wr, Wg, Wu, Wd, 4, "relu", False, True, np.array([1, 0, 1, -1, 2]))
    p = np.exp(X @ Wr)
    p /= p.sum(1, keepdims=True)
    want = sum(p[:, e:e + 1] * OH.ffn_forward(X, Wg[e], Wu[e], Wd[e], "relu", False) for e in range(4))
    want[[1, 3]] = 0
    close(Y, want, 1e-12)
    assert (idx[[1, 3]] == -1).all() and (w[[1, 3]] == 0).all()
    idx, w = OM.route(np.zeros((1, 6)), Wr, 3, False)
    assert idx.tolist() == [[0, 1, 2]] and np.allclose(w, 0.25)
    idx, w = OM.route(X, Wr, 2, False)
    assert np.allclose(w, np.take_along_axis(p, idx, 1)) and (w[:, 0] >= w[:, 1]).all()


def params(hg, d=128, f=384, E=8, top=2, dt=1, act=3, Wr=FAR[8], Wg=FAR[9], Wu=FAR[10], Wd=FAR[11]):  # noqa: F811
    return ctypes.byref(hg.hg_moe_params(d, f, E, top, dt, act, 0, 1, Wr, Wg, Wu, Wd))


def test_sizes(hg):  # noqa: F811
    so = hg.lib()
    b = ctypes.c_size_t()

    def query(n=10, **k):
        return so.hg_moe_workspace_size(params(hg, **k), n, ctypes.byref(b))

    assert query() == 0 and b.value > 4 * 16 * 128 * 10
    assert query(0) == 0 and b.value == 0
    small = query(1) or b.value
    assert query(1024) == 0 and b.value > small
    assert query(1025) == 2 and query(d=96) == 2 and query(dt=2) == query(dt=-1) == 2
    assert query(-1) == query(f=0) == query(f=12) == query(f=16392) == query(E=0) == query(E=257) == 1
    assert query(top=0) == query(top=9, E=16) == query(top=3, E=2) == query(act=4) == query(act=-1) == 1
    assert so.hg_moe_workspace_size(None, 1, ctypes.byref(b)) == so.hg_moe_workspace_size(params(hg), 1, None) == 1


def test_refusals(hg):  # noqa: F811
    so = hg.lib()

    def fwd(n=10, X=FAR[0], live=None, Y=FAR[1], e=FAR[2], w=FAR[3], scratch=FAR[4], **k):
        return so.hg_moe_fwd(params(hg, **k), X, live, n, Y, e, w, scratch, None)

    assert fwd(n=-1) == fwd(f=4) == 1 and fwd(d=32) == fwd(n=1025) == 2
    assert fwd(n=0, X=None, Y=None, scratch=None) == 0
    assert fwd(X=None) == fwd(Y=None) == fwd(scratch=None) == 1
    assert fwd(Wr=None) == fwd(Wg=None) == fwd(Wu=None) == fwd(Wd=None) == 1
    assert fwd(Wr=A + 8) == fwd(Wg=A + 8) == fwd(Wu=A + 2) == fwd(Wd=A + 4) == 1
    assert fwd(X=A + 8) == fwd(Y=A + 4) == fwd(scratch=A + 16) == fwd(live=A + 2) == fwd(e=A + 1) == fwd(w=A + 2) == 1
    # an output in another array's place, or part of it
    for i in (0, 2, 3, 4, 8, 9, 10, 11):
        assert fwd(Y=FAR[i]) == 1
    assert fwd(Y=FAR[0] + 10 * 256 - 16) == fwd(Y=FAR[9] + 8 * 128 * 384 * 2 - 16) == fwd(Y=FAR[5], live=FAR[5]) == 1
    assert fwd(scratch=FAR[0]) == fwd(scratch=FAR[10]) == fwd(scratch=FAR[2]) == 1
    assert fwd(e=FAR[0]) == fwd(e=FAR[3]) == fwd(e=FAR[11] + 64) == fwd(w=FAR[8]) == fwd(w=FAR[5], live=FAR[5]) == 1


def test_binding_refuses_what_it_would_read_wrongly(hg):  # noqa: F811
    Wr, Wg, Wd = torch.zeros(64, 2), torch.zeros(2, 64, 8), torch.zeros(2, 8, 64)
    with pytest.raises(ValueError, match="device memory"):
        hg.MoeParams(Wr, Wg, Wg, Wd, 1)
    with pytest.raises(ValueError, match="W_router must be"):
        hg.MoeParams(Wr.T, Wg, Wg, Wd, 1)
    with pytest.raises(ValueError, match="storage types"):
        hg.MoeParams(*(t.half() for t in (Wr, Wg, Wg, Wd)), 1)
