"""Long memories of the gated linear recurrence: gates that hardly change over tens of thousands of positions, where a
rounding of one sign at every position would add up.

Bounds, with u = half a step of the storage type, s = 2^-24, M and A the sums of the absolute terms of the state and of R:
  z                 (2 |a| + 12) s of itself: the logit's product (2 |a| s, constant and rounding), exponential, quotient
                    and sum.  A state, and z R, follow it by at most as much of M, and of z A.
  a run's B and Q   a tile's sums of at most 16 positions, 16 runs and two more: two, three and three roundings each, 86 s
                    of themselves, and what they are off by is forgotten as fast as it is added: 86 s M.  A chain that is
                    kept in two numbers rounds what at most 16 positions add: 16 s M, and at the sum 2 s M.
  a tile's step     one rounding of the state: T / 128 s M for tiles of at least 128 positions.  (Chains in bf16 round it at
                    every position: T s M.)
Together e = (T / 128 + 2 |a| + 140) s of M or A.  dx adds the product's rounding (40 s as elsewhere); dg is off by R's and
the difference's errors, and by products: (2 e + 200 s) of z (1 - z) A (|x| + M).
"""
import numpy as np
import pytest
import torch

from oracle import recur as OR
from tests.gpu_util import dev, lib, need_gpu, tdtype
from tests.test_gpu_history import F32, U, draw, f64, nans, near
from tests.test_gpu_recur import params, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("logit", [-9.0, -11.5, -13.75])
@pytest.mark.parametrize("n,T", [(3, 32768), (1, 5000), (20000, 8192)])
def test_constant_gates(dt, logit, n, T):
    """Rows that repeat, one for all positions and histories (strides of zero): few histories, whose time is split, and many,
    each a chain.  A state that is its input stays where it is."""
    need_gpu()
    hg = lib()
    td, d = tdtype(dt), 8
    rng = np.random.default_rng(int(-logit))
    g = (logit + np.arange(d) / 32).astype(np.float32)  # (as bf16 some are equal)
    x, dy, h, dh = (draw(rng, dt, d) for _ in range(4))
    h[3] = x[3]
    h[4], x[5], dy[6] = 0, 0, 0
    G, X, DY = (dev(v, td).expand(n, T, d) for v in (g, x, dy))
    H, DH = (dev(v).expand(n, d).contiguous() for v in (h, dh))
    o = run(hg, hg.RecurParams(d=d, dtype=td), td, X, G, None, H, DY, DH, n, T, d)
    for k in ("y", "dx", "dg", "h", "dh"):
        assert (o[k] == o[k][:1]).all(), k  # the histories are one
    a = f64(G[0, 0].float().cpu().numpy())
    x, dy, h, dh = (f64(v) for v in (x, dy, h, dh))
    z, keep = 1 / (1 + np.exp(-a)), 1 / (1 + np.exp(a))
    lk = np.log1p(-z)
    t = np.arange(T)[:, None]
    steps = T if dt == "bf16" and n > 1000 else T / 128
    e = (steps + 2 * np.abs(a).max() + 140) * F32
    M = np.maximum(np.abs(x), np.abs(h))
    state = lambda p: x + (h - x) * np.exp(p * lk)  # noqa: E731  after p positions
    near(o["y"][0], state(t + 1), M, (U[dt], e), "y")
    near(o["h"][0], state(T), M, (F32, e), "h_out")
    R = lambda w, last: w * -np.expm1((T - t) * lk) / z + last * np.exp((T - 1 - t) * lk)  # noqa: E731
    r, A = R(dy, dh), R(np.abs(dy), np.abs(dh))
    near(o["dx"][0], z * r, z * A, (U[dt], e + 40 * F32), "dx")
    near(o["dh"][0], keep * r[0], keep * A[0], (F32, e), "dh_in")
    near(o["dg"][0], r * (x - state(t)) * z * keep, A * (np.abs(x) + M) * z * keep, (U[dt], 2 * e + 200 * F32), "dg")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T", [600, 32768])
def test_gates_of_small_spread(dt, T):
    """Inputs as they come, gates about a bias of -9 to -13, against the definition position by position."""
    need_gpu()
    hg = lib()
    td, n, d = tdtype(dt), 2, 16
    rng = np.random.default_rng(T)
    x, dy = draw(rng, dt, n, T, d), draw(rng, dt, n, T, d)
    g = draw(rng, dt, n, T, d, scale=0.25)
    b = draw(rng, dt, d, scale=0.0) - np.linspace(9, 13, d).astype(np.float32)
    b = f64(dev(b, td).float().cpu().numpy())
    h, dh = rng.standard_normal((2, n, d)).astype(np.float32)
    o = run(hg, params(hg, b.astype(np.float32), d, td), td, dev(x, td), dev(g, td), None, dev(h), dev(dy, td), dev(dh), n, T,
            d)
    e = (T / 128 + 2 * (13 + 0.25 * 6) + 140) * F32
    y, last, _, most = OR.forward(f64(x), f64(g), b, None, f64(h))
    near(o["y"], y, np.broadcast_to(most[:, None], y.shape), (U[dt], e), "y")
    near(o["h"], last, most, (F32, e), "h_out")
    want, mag = OR.backward(f64(x), f64(g), f64(dy), b, None, f64(h), f64(dh))
    near(o["dx"], want["dx"], mag["dx"], (U[dt], e + 40 * F32), "dx")
    near(o["dg"], want["dg"], mag["dg"], (U[dt], 2 * e + 200 * F32), "dg")
    near(o["dh"], want["dh_in"], mag["dh_in"], (F32, e), "dh_in")


@pytest.mark.parametrize("T", [1, 40, 700])
def test_biases_and_logits_that_cancel(T):
    """fp32: a gate is that of the sum of logit and bias, to (3 |a| + 12) s of itself (the sum's rounding, and as above),
    however large the two are.  With inputs of one and a state of zero, y_t = 1 - (1 - z)^(t + 1), and a run's own roundings
    (100 s)."""
    need_gpu()
    hg = lib()
    pairs = [(60.3, -60.3), (-77.3, -3.1), (-3.1, -77.3), (1000.1, -1000.1), (-1000.1, 990.0), (70.7, -75.2), (5e8, -5e8),
             (-1e6, 1e6 + 4)]
    g, b = (np.array(v, np.float32) for v in zip(*pairs))
    d, n = 8, 2
    p = hg.RecurParams(dev(b))
    G, X = dev(g).expand(n, T, d), torch.ones(n, T, d, device="cuda")
    y, h = nans((n, T, d), torch.float32), nans((n, d), torch.float32)
    hg.hg_recur_fwd(p, X, G, None, None, y, h, None)
    a = f64(g) + f64(b)
    z = 1 / (1 + np.exp(-a))
    t = np.arange(1, T + 1)[:, None]
    want = -np.expm1(t * np.log1p(-z))
    rel = (3 * np.abs(a) + 112) * F32
    assert (np.abs(y.double().cpu().numpy() - want) <= rel * want).all()
    # the state goes through whole tiles, a row through its own run: other sums, each within the same bound
    assert (np.abs(h.double().cpu().numpy() - want[-1]) <= rel[None] * want[-1]).all()
    s = torch.zeros(n, d, device="cuda")
    hg.hg_recur_step(p, X[:, 0], G[:, 0], None, s, y[:, 0])
    assert (np.abs(s.double().cpu().numpy() - z) <= (3 * np.abs(a) + 12) * F32 * z).all()
    # and the gradients: of ones at the end z (1 - z)^(T - 1 - t) is left, whose logarithm follows z by T - t times its share
    saved, scratch = (torch.empty(v, dtype=torch.uint8, device="cuda") for v in hg.hg_recur_workspace_size(p, n, T))
    hg.hg_recur_fwd(p, X, G, None, None, y, h, saved)
    dx, dg, dh = nans((n, T, d), torch.float32), nans((n, T, d), torch.float32), nans((n, d), torch.float32)
    one = torch.ones(n, d, device="cuda")
    hg.hg_recur_bwd(p, X, G, None, None, saved, torch.zeros(n, T, d, device="cuda"), one, dx, dg, dh, None, None)
    left = np.exp((T - t) * np.log1p(-z))
    off = rel * (1 + 2 * (T - t) * z)
    assert (np.abs(dx.double().cpu().numpy() - z * left) <= (off + rel) * z * left + 1e-37).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,d", [(40, 12, 64), (300, 70, 64), (3, 900, 40)])
def test_biases_near_the_largest_number(dt, n, T, d):
    """A bias of +-3e38 is one that no logit moves, with ragged histories: z is 1 or 0."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    rng = np.random.default_rng(7)
    x, g, dy = (draw(rng, dt, n, T, d) for _ in range(3))
    h, dh = rng.standard_normal((2, n, d)).astype(np.float32)
    lens = rng.integers(0, T + 1, n).astype(np.int32)
    lens[0], lens[-1] = 0, T
    b = np.zeros(d, np.float32)
    b[1], b[2] = 3e38, -3e38
    X, H, L = dev(x, td), dev(h), dev(lens)
    o = run(hg, hg.RecurParams(dev(b, td)), td, X, dev(g, td), L, H, dev(dy, td), dev(dh), n, T, d)
    live = torch.arange(T, device="cuda") < L[:, None]
    assert all(torch.isfinite(v).all() for v in o.values())
    assert torch.equal(o["y"][..., 2], (H[:, None, 2] * live).to(td)) and torch.equal(o["h"][:, 2], H[:, 2])
    # an open gate leaves the value to a step of it, or in bf16 of what was there (x, state and their difference: 6 steps)
    most = max(np.abs(x).max(), np.abs(h).max())
    want = X[..., 1].double() * live
    assert ((o["y"][..., 1].double() - want).abs() <= U[dt] * want.abs() + (6 * F32 * most if dt == "bf16" else 0)).all()
    assert (o["dx"][..., 2] == 0).all() and (o["dg"][..., 1:3] == 0).all() and (o["db"][1:3] == 0).all()
