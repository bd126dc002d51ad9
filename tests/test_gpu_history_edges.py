"""Edges of the history encoder's operators: values that are infinite, NaN or far from one, many rows a CTA, and bounds
as tight as the kernels' sums.  Helpers and the way tolerances are written: test_gpu_history.py."""
import numpy as np
import pytest
import torch

from hgsynth import bf16_round
from oracle import history as OH
from tests.gpu_util import dev, lib, need_gpu, tdtype
from tests.test_gpu_history import (F32, LD, U, decay_problem, decay_rel, f64, host, nans, near, past, rot_problem,
                                    rot_rel, strided)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ gated block
GATES = np.array([0, 0.5, 2, 3.5, 7, 9, 20, 100, 300, 2.0**18, 1e6, 2.0**22, 1e10, 1e14, 1e20, 1e30], np.float32)


def gates_problem(dt):
    """G = the gates, U = 1, dH = dY: rows of gates in features 0..31 (feature 63 is one), unit weights."""
    vals = np.concatenate([GATES, -GATES])
    if dt == "bf16":
        vals = bf16_round(vals)
    n, d = 37, 64
    X, dY = np.zeros((n, d), np.float32), np.zeros((n, d), np.float32)
    X[:, :32] = vals[(np.arange(32) + np.arange(n)[:, None]) % 32]
    X[:, 63] = 1
    dY[:, :32] = np.where((np.arange(32) + np.arange(n)[:, None]) % 3 == 0, -0.75, 1.25)
    Wg, Wu, Wd = np.zeros((d, d), np.float32), np.zeros((d, d), np.float32), np.eye(d, dtype=np.float32)
    Wg[np.arange(32), np.arange(32)] = 1
    Wu[63] = 1
    return X, Wg, Wu, Wd, dY


def gates_run(hg, dt, act):
    """Y, dX and the weights' gradients of gates_problem, and what act and act' are there."""
    td = tdtype(dt)
    X, Wg, Wu, Wd, dY = gates_problem(dt)
    n, d = X.shape
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)), act=act)
    work = torch.empty(max(hg.hg_ffn_workspace_size(p, n)), dtype=torch.uint8, device="cuda")
    Y, dX = nans((n, d), td), nans((n, d), td)
    g = {k: nans((d, d), torch.float32) for k in ("W_gate", "W_up", "W_down")}
    hg.hg_ffn_fwd(p, dev(X, td), Y, work)
    hg.hg_ffn_bwd(p, dev(X, td), dev(dY, td), dX, g, work)
    X, dY = f64(X), f64(dY)
    A, dA = OH.act(np.clip(X, -1e4, 1e4), act)
    if act != "none":  # beyond 1e4: x or 0, 1 or 0
        big = np.abs(X) > 1e4
        A, dA = np.where(big, np.maximum(X, 0), A), np.where(big, (X > 0) * 1.0, dA)
    else:
        A = X
    return X, dY, A, dA, Y, dX, g


g32 = slice(0, 32)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu", "none"])
def test_values_of_gates_of_every_size(dt, act):
    """act of gates from 0 to 1e30 of either sign.  G, U and dH are exact and a sum has one term: the functions within
    30 steps of |x|, in bf16 H rounded once; dW_up sums 37 rows, in bf16 of two terms."""
    need_gpu()
    X, dY, A, _, Y, _, g = gates_run(lib(), dt, act)
    near(Y[:, g32], A[:, g32], np.abs(X[:, g32]), (U[dt], 30 * F32), "Y")
    s = (2.0**-16 if dt == "bf16" else 0) + (30 + 37) * F32
    near(g["W_up"][63, g32], (dY * A).sum(0)[g32], (np.abs(dY) * np.abs(X)).sum(0)[g32], (0, s), "W_up")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu", "none"])
def test_derivatives_of_gates_of_every_size(dt, act):
    """act' of the same gates: that of a large one is 1 or 0.  Within 70 steps of 1 (a slope below 2.3 times 30 steps
    where it is neither 0 nor 1), in bf16 dG rounded once; dW_gate sums 37 rows, in bf16 of two terms."""
    need_gpu()
    X, dY, _, dA, _, dX, g = gates_run(lib(), dt, act)
    near(dX[:, g32], (dY * dA)[:, g32], np.abs(dY[:, g32]), (U[dt], 70 * F32), "dX")
    s = (2.0**-16 if dt == "bf16" else 0) + (70 + 37) * F32
    near(g["W_gate"][:, g32], X.T @ (dY * dA)[:, g32], np.abs(X).T @ np.abs(dY[:, g32]), (0, s), "W_gate")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu", "none"])
def test_a_gate_that_is_nan_is_seen(dt, act):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    X, Wg, Wu, Wd, dY = gates_problem(dt)
    X[:, :32] = np.clip(X[:, :32], -4, 4)
    Wg[63, 40] = np.nan  # one hidden feature's gate, of every row
    n, d = X.shape
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)), act=act)
    work = torch.empty(max(hg.hg_ffn_workspace_size(p, n)), dtype=torch.uint8, device="cuda")
    Y, dX = torch.zeros(n, d, dtype=td, device="cuda"), torch.zeros(n, d, dtype=td, device="cuda")
    g = {k: torch.zeros(d, d, device="cuda") for k in ("W_gate", "W_up", "W_down")}
    hg.hg_ffn_fwd(p, dev(X, td), Y, work)
    assert torch.isnan(Y).all()  # the feature is a term of every column
    dY[:, 40] = 1
    hg.hg_ffn_bwd(p, dev(X, td), dev(dY, td), dX, g, work)
    assert torch.isnan(dX).all() and torch.isnan(g["W_up"][:, 40]).all() and torch.isnan(g["W_down"][40]).all()


def test_ffn_input_gradient_alone_needs_no_scratch_in_bf16():
    need_gpu()
    hg = lib()
    for td in (torch.bfloat16, torch.float32):
        gen = torch.Generator(device="cuda").manual_seed(2)
        new = lambda *s: torch.randn(*s, device="cuda", generator=gen).mul_(0.25).to(td)  # noqa: E731
        X, dY, p = new(150, 64), new(150, 64), hg.FfnParams(new(64, 72), new(64, 72), new(72, 64))
        work = torch.empty(hg.hg_ffn_workspace_size(p, 150)[1], dtype=torch.uint8, device="cuda")
        a, b = nans((150, 64), td), nans((150, 64), td)
        hg.hg_ffn_bwd(p, X, dY, a, None, work)
        if td == torch.bfloat16:
            hg.hg_ffn_bwd(p, X, dY, b, None, None)
            assert torch.equal(a, b)
        else:
            with pytest.raises(ValueError, match="bytes are needed"):
                hg.hg_ffn_bwd(p, X, dY, b, None, None)


def test_long_sums_of_one_sign_do_not_shrink():
    """Weight gradients of positive rows in one share of 157 row tiles (d 64, 152 chunks of hidden features).  Tensor
    additions cut their results (2^-23 at most): 4 for each of U and dH (or G), 16 for a tile's rows, so the mean of the
    relative errors is above -24 2^-23 = -2.9e-6.  The rest is rounded to nearest and does not lean: 157 tiles at 2^-24,
    the two terms at 2^-17; all together below 2e-5 in any one value."""
    need_gpu()
    hg = lib()
    n, d, f, td = 20_000, 64, 152 * 64, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.rand(*s, device="cuda", generator=gen).add_(0.5).to(td)  # noqa: E731
    X, dY, Wg, Wu, Wd = new(n, d), new(n, d), new(d, f), new(d, f), new(f, d)
    p = hg.FfnParams(Wg, Wu, Wd, act="none")
    g = {k: nans(w.shape, torch.float32) for k, w in (("W_gate", Wg), ("W_up", Wu), ("W_down", Wd))}
    hg.hg_ffn_bwd(p, X, dY, None, g, torch.empty(hg.hg_ffn_workspace_size(p, n)[1], dtype=torch.uint8, device="cuda"))
    X, dY, Wg, Wu, Wd = (x.double() for x in (X, dY, Wg, Wu, Wd))
    G, U_, dH = X @ Wg, X @ Wu, dY @ Wd.T
    for key, want in (("W_gate", X.T @ (dH * U_)), ("W_up", X.T @ (dH * G)), ("W_down", (G * U_).T @ dY)):
        off = g[key].double() / want - 1
        assert off.abs().max() < 2e-5, (key, off.abs().max())
        assert abs(off.mean()) < 4e-6, (key, off.mean())


# ------------------------------------------------------------------------------------------------- decay
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("T,h,dh", [(40, 2, 32), (37, 1, 16), (40, 2, 64), (20, 1, 128), (900, 1, 64)])
def test_decay_is_causal_whatever_the_values(dt, bad, T, h, dh):
    """An infinity or NaN at one position of one head: o, dq at earlier positions and dk, dv at later ones are what they
    are without it, and so are the other heads and, where it is a value feature, the other columns."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    at = [0, 5, 7, 15, 16, 23, T - 1]
    n = len(at)
    q, k, v, do, lens, S, dS = decay_problem(dt, n, T, h, dh, T + dh, False, True)
    lens = np.full(n, T, np.int32)
    lens[2] = 9
    at = np.minimum(at, lens - 1)
    c = np.float64(np.float32(0.3))
    ld = np.array([-0.05, -0.4], np.float32)[:h]
    p = hg.DecayParams(dev(ld), dh, td, scale=0.3)
    work = torch.empty(max(hg.hg_decay_workspace_size(p, n, T)), dtype=torch.uint8, device="cuda")
    args = [f64(x) for x in (q, k, v)] + [f64(ld), c]
    names = ("o", "last", "dq", "dk", "dv", "dS")
    want, terms = ({**dict(zip(names, OH.decay_forward(*args, lens, f64(S), magnitude=m))),
                    **dict(zip(names[2:], OH.decay_backward(*args, f64(do), lens, f64(S), f64(dS), magnitude=m)))}
                   for m in (False, True))
    t = np.arange(T)[None]
    before, after, own = t < at[:, None], t > at[:, None], t == at[:, None]
    every, none = np.ones((n, T), bool), np.zeros((n, T), bool)
    # which positions of the poisoned head an array's bad value leaves alone, and whether it is held to a column
    reach = {"q": dict(o=~own, dq=every, dk=(after, True), dv=after),
             "k": dict(o=before, dq=(before, True), dk=every, dv=~own),
             "v": dict(o=(before, True), dq=before, dk=~own, dv=every),
             "do": dict(o=every, dq=~own, dk=after, dv=(after, True))}
    for name, clean in reach.items():
        x = {"q": q, "k": k, "v": v, "do": do}
        x[name] = x[name].copy()
        x[name][np.arange(n), at, 0, 3] = bad * (1 if name != "k" else -1)
        Q, K, V, DO = (strided(past(y, lens), td) for y in x.values())
        o = nans((n, T, h, dh), td)
        hg.hg_decay_fwd(p, Q, K, V, dev(lens), dev(S), o, None, work)
        g = [nans((n, T, h, dh), td) for _ in range(3)] + [nans((n, h, dh, dh), torch.float32)]
        hg.hg_decay_bwd(p, Q, K, V, dev(lens), dev(S), DO, dev(dS), *g, work)
        for out, got in zip(("o", "dq", "dk", "dv"), (o, *g[:3])):
            rows = clean[out]
            rows, column = rows if isinstance(rows, tuple) else (rows, False)
            good = np.ones((n, T, h, dh), bool)
            good[:, :, 0] = rows[..., None]
            if column:
                good[:, :, 0, np.arange(dh) != 3] = True
            got = host(got)
            live = np.broadcast_to((t < lens[:, None])[:, :, None, None], good.shape)
            assert not np.isfinite(got[~good & live]).any(), (name, out)
            assert (got[~live] == 0).all()
            near(torch.from_numpy(np.where(good, got, 0)), np.where(good, want[out], 0), np.where(good, terms[out], 0),
                 decay_rel(dt, T, dh, "rows"), (name, out))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("swap", [False, True])
def test_outputs_between_inputs_in_the_same_rows(dt, swap):
    """Every array a slice of one wide row (or positions outside, sequences inside): accepted, the bits of arrays apart,
    and nothing else written."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    n, T, h, dh = 5, 21, 2, 32
    q, k, v, do, lens, S, dS = decay_problem(dt, n, T, h, dh, 4, True, True)
    p, r = hg.DecayParams(dev(LD[:h]), dh, td), hg.QkRotParams(None, None, h, h, d_h=dh, dtype=td)
    wide = nans((T, n, 11, h, dh) if swap else (n, T, 11, h, dh), td)
    view = wide.transpose(0, 1) if swap else wide
    x = [view[:, :, i] for i in (0, 2, 4, 6)]
    out = [view[:, :, i] for i in (1, 3, 5, 7)]
    for a, b in zip(x, (q, k, v, do)):
        a.copy_(dev(b, td))
    want = [nans((n, T, h, dh), td) for _ in range(4)]
    for y, o in ((x, out), ([a.contiguous() for a in x], want)):
        hg.hg_decay_fwd(p, *y[:3], dev(lens), dev(S), o[0], None, None)
        hg.hg_decay_bwd(p, *y[:3], dev(lens), dev(S), y[3], dev(dS), *o[1:], None, None)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(torch.equal(a, dev(b, td)) for a, b in zip(x, (q, k, v, do))) and torch.isnan(view[:, :, 8:]).all()
    rows = [wide.view(n * T, 11, h, dh)[:, i] for i in (8, 9, 0, 2)]
    hg.hg_qkrot_fwd(r, rows[2], rows[3], None, rows[0], rows[1])
    a, b = nans((n * T, h, dh), td), nans((n * T, h, dh), td)
    hg.hg_qkrot_fwd(r, rows[2].contiguous(), rows[3].contiguous(), None, a, b)
    assert torch.equal(rows[0], a) and torch.equal(rows[1], b)
    hg.hg_qkrot_fwd(r, rows[2], rows[3], None, rows[2], rows[3])  # in place, side by side
    assert torch.equal(rows[2], a) and torch.equal(rows[3], b) and torch.isnan(view[:, :, 10]).all()
    with pytest.raises(hg.HGError, match="overlap"):
        hg.hg_decay_fwd(p, *x[:3], dev(lens), None, view[:, :, 4:6].flatten(2, 3)[:, :, 1:3], None, None)
    with pytest.raises(hg.HGError, match="overlap"):
        hg.hg_qkrot_fwd(r, rows[2][:-1], rows[3][:-1], None, rows[2][1:], rows[3][:-1])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,dh", [(1, 16), (1, 32), (1, 128), (2, 64), (2, 32)])
def test_decay_states_are_fp32_sums(dt, T, dh):
    """States of one and two positions.  A term: its factor c gamma^t (the product 1, 2^x and x 6), the product with it
    1, each of three tensor additions cut at 2^-23 (6), a last factor (7), and T such terms: 21 T steps of 2^-24 of
    their sizes.  Two bf16 numbers for a scaled value, in place of three, would be seen: planted in the oracle here."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    n, h = 3, 2
    q, k, v, do, *_ = decay_problem(dt, n, T, h, dh, T + dh, False, False)
    c, ld = np.float64(np.float32(0.3)), np.array([0.0, -0.3], np.float32)
    p = hg.DecayParams(dev(ld), dh, td, scale=0.3)
    x = [dev(y, td) for y in (q, k, v)]
    o, last, dlast = nans((n, T, h, dh), td), nans((n, h, dh, dh), torch.float32), nans((n, h, dh, dh), torch.float32)
    work = torch.empty(max(hg.hg_decay_workspace_size(p, n, T)), dtype=torch.uint8, device="cuda")
    hg.hg_decay_fwd(p, *x, None, None, o, last, work)
    hg.hg_decay_bwd(p, *x, None, None, dev(do, td), None, *(nans((n, T, h, dh), td) for _ in range(3)), dlast, work)
    args = [f64(y) for y in (q, k, v)] + [f64(ld), c]
    rel = (0, 21 * T * F32)
    near(last, OH.decay_forward(*args)[1], OH.decay_forward(*args, magnitude=True)[1], rel, "state")
    want, size = (OH.decay_backward(*args, f64(do), magnitude=m)[3] for m in (False, True))
    near(dlast, want, size, rel, "state's gradient")
    y = (c * f64(do)).astype(np.float32)  # the planted mistake
    hi = bf16_round(y)
    two = f64(hi) + f64(bf16_round(y - hi))
    off = OH.decay_backward(*args[:4], 1.0, two)[3]
    assert (np.abs(off - want) > rel[1] * size).any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_every_call_repeats_its_bits(dt):
    """Ragged histories that are claimed, segments, shares of rows: no sum's order depends on the run."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    n, T, h, dh = 60, 300, 4, 32
    q, k, v, do, lens, S, dS = decay_problem(dt, n, T, h, dh, 1, True, True)
    p = hg.DecayParams(dev(LD[:h]), dh, td, scale=0.25)
    r = hg.QkRotParams(torch.ones(dh, dtype=td, device="cuda"), torch.ones(dh, dtype=td, device="cuda"), h, h)
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = [torch.randn(*s, device="cuda", generator=gen).mul_(0.1).to(td) for s in ((128, 200), (128, 200), (200, 128))]
    f = hg.FfnParams(*w)
    Q, K, V, DO = (dev(x, td) for x in (q, k, v, do))
    need = max(*hg.hg_decay_workspace_size(p, n, T), *hg.hg_ffn_workspace_size(f, n * T),
               hg.hg_qkrot_workspace_size(r, n * T))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    runs = []
    for _ in range(4):
        work.random_(0, 255)
        new = lambda *s, dtype=td: nans(s, dtype)  # noqa: E731
        out = [new(n, T, h, dh) for _ in range(6)] + [new(n, h, dh, dh, dtype=torch.float32) for _ in range(2)]
        hg.hg_decay_fwd(p, Q, K, V, dev(lens), dev(S), out[0], out[6], work)
        hg.hg_decay_bwd(p, Q, K, V, dev(lens), dev(S), DO, dev(dS), *out[1:4], out[7], work)
        rows = [x.view(n * T, h, dh) for x in (Q, K, DO, V, out[4], out[5])]
        g = {"gamma_q": new(dh, dtype=torch.float32), "gamma_k": new(dh, dtype=torch.float32)}
        hg.hg_qkrot_bwd(r, rows[0], rows[1], None, *rows[2:], g, work)
        y, dx = new(n * T, 128), new(n * T, 128)
        fg = {x: nans(z.shape, torch.float32) for x, z in zip(("W_gate", "W_up", "W_down"), w)}
        hg.hg_ffn_fwd(f, Q.view(n * T, 128), y, work)
        hg.hg_ffn_bwd(f, Q.view(n * T, 128), DO.view(n * T, 128), dx, fg, work)
        runs.append([*out, *g.values(), y, dx, *fg.values()])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


# ---------------------------------------------------------------------------------------------- rotation
# A resident set of CTAs (three an SM, two backward) takes these rows in three rounds and more, the last one ragged:
# heads in fours, in twos and odd, that divide a CTA's groups and that do not.
MANY = [("bf16", 80_001, 2, 2, 16), ("bf16", 25_003, 2, 1, 64), ("bf16", 10_007, 5, 1, 64), ("bf16", 9_001, 5, 2, 64),
        ("bf16", 13_003, 4, 0, 128), ("f32", 31_001, 2, 2, 32), ("f32", 21_001, 3, 0, 64), ("f32", 5_003, 5, 1, 128),
        ("f32", 3_001, 6, 5, 128), ("bf16", 26_001, 3, 3, 32)]


@pytest.mark.parametrize("dt,n,hq,hk,dh", MANY)
def test_qkrot_of_many_rows(dt, n, hq, hk, dh):
    """The bits of the rows in small batches, in which a group of lanes has one row, in place too; the gains' sums are
    those of runs of at most ten rows a group, 256 groups a CTA and 57 CTAs a thread."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    rng, q, k, gq, gk, pos = rot_problem(dt, n, hq, hk, dh, n, True)
    how = (dh, 1000.0, 1e-4, hq % 2 == 1)
    p = hg.QkRotParams(dev(gq, td), dev(gk, td), hq, hk, rot=dh, base=1000.0, eps=1e-4, interleaved=how[3])
    dy = [dev(x, td) for x in (rng.standard_normal((n, hq, dh)), rng.standard_normal((n, hk, dh)))]
    Q, K, P = strided(q, td), strided(k, td), dev(pos)
    work = torch.empty(hg.hg_qkrot_workspace_size(p, n), dtype=torch.uint8, device="cuda")
    some = lambda x, s: x[s] if hk else None  # noqa: E731
    out = [nans((n, hq, dh), td), nans((n, hk, dh), td), nans((n, hq, dh), td), nans((n, hk, dh), td)]
    small = [x.clone() for x in out]
    g = {"gamma_q": nans((dh,), torch.float32), "gamma_k": nans((dh,), torch.float32)}

    def both(to, s, grads, work):
        hg.hg_qkrot_fwd(p, Q[s], some(K, s), P[s], to[0][s], some(to[1], s))
        hg.hg_qkrot_bwd(p, Q[s], some(K, s), P[s], dy[0][s], some(dy[1], s), to[2][s], some(to[3], s), grads, work)

    both(out, slice(0, n), g, work)
    for i in range(0, n, 997):
        both(small, slice(i, min(i + 997, n)), {}, work)
    assert all(torch.isfinite(x).all() and torch.equal(x, y) for x, y in zip(out, small))
    e = rot_rel(dt)[1] + (10 + 256 + 57 + 8) * F32
    for x, gain, d, key in ((q, gq, dy[0], "gamma_q"), (k, gk, dy[1], "gamma_k")):
        x, gain, d = f64(x), f64(gain), host(d)
        a, b = OH.pair_index(dh, how[3])
        t = np.abs(d)
        t[..., a] = t[..., b] = t[..., a] + t[..., b]
        u = np.abs(x) / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-4)
        near(g[key], OH.qkrot_backward(x, gain, pos, *how, d)[1], (t * u).sum((0, 1)), (0, e), key)
    inq, ink = Q.contiguous(), K.contiguous()
    hg.hg_qkrot_fwd(p, inq, ink if hk else None, P, inq, ink if hk else None)
    assert torch.equal(inq, out[0]) and torch.equal(ink, out[1])
    dq, dk = dy[0].clone(), dy[1].clone()
    hg.hg_qkrot_bwd(p, Q, K if hk else None, P, dq, dk if hk else None, dq, dk if hk else None, {}, work)
    assert torch.equal(dq, out[2]) and torch.equal(dk, out[3])
