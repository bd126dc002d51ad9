"""History encoder's operators (hg_qkrot_*, hg_decay_*, hg_ffn_*) through the C ABI against the fp64 oracle.

Tolerances, element by element, with u = half a step of the storage type (2^-24 fp32, 2^-8 bf16):
  |got - want| <= u |want| + r A + e A,  A = the sum of the absolute values of the result's terms,
where r counts the roundings of factors to the storage type inside the kernel (0 in fp32) and e the fp32 sums and
functions: a sum of m terms is within m 2^-24 A in any order; each test gives its own r and e.
"""
import numpy as np
import pytest
import torch

from hgsynth import bf16_round
from oracle import history as OH
from tests.gpu_util import dev, lib, need_gpu, tdtype

pytestmark = pytest.mark.gpu

U = {"f32": 2.0**-24, "bf16": 2.0**-8}
F32 = 2.0**-24


def draw(rng, dt, *shape, scale=1.0):
    x = (rng.standard_normal(shape) * scale).astype(np.float32)
    return bf16_round(x) if dt == "bf16" else x


def f64(x):
    return None if x is None else np.asarray(x, np.float64)


def host(t):
    return t.detach().double().cpu().numpy()


def nans(shape, dtype):
    return torch.full(tuple(shape), float("nan"), dtype=dtype, device="cuda")


def near(got, want, terms, rel, what):
    got = host(got)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - (rel[0] * np.abs(want) + rel[1] * terms + 1e-30)
    assert over.max(initial=-1) <= 0, (what, over.max(), np.abs(got - want).max())


def strided(x, td, pad_heads=1):
    """x [..., heads, d_h] on the device as a slice of a wider row."""
    wide = nans((*x.shape[:-2], x.shape[-2] + 2 * pad_heads, x.shape[-1]), td)
    view = wide[..., pad_heads:pad_heads + x.shape[-2], :]
    view.copy_(dev(x, td))
    return view


# ---------------------------------------------------------------------------------------------- rotation
def rot_problem(dt, n, hq, hk, dh, seed, far):
    rng = np.random.default_rng(seed)
    q, k = draw(rng, dt, n, hq, dh), draw(rng, dt, n, hk, dh)
    gq, gk = 1 + draw(rng, dt, dh, scale=0.25), 1 + draw(rng, dt, dh, scale=0.25)
    if dt == "bf16":
        gq, gk = bf16_round(gq), bf16_round(gk)
    pos = rng.integers(-(1 << 31) + 1, 1 << 31, n) if far else rng.integers(0, 400, n)
    return rng, q, k, gq, gk, pos


# r = 0: one rounding at the end.  e: the norm's sum (128 terms, half of their error in the root), the root, two
# products and the turn: below 80 steps; the angle: 4e-7 + 2^-21 (bf16's sine) of A.
def rot_rel(dt):
    return U[dt], 160 * F32 + 4e-7 + (2.0**-20 if dt == "bf16" else 0)


def rot_terms(f, x, gamma, pos, *how):
    """|a| + |b| of a turned pair: the largest turn of the absolute values."""
    y = np.abs(x) / np.sqrt((x * x).mean(-1, keepdims=True) + how[2]) * np.abs(gamma)
    a, b = OH.pair_index(how[0], how[3])
    t = y.copy()
    t[..., a] = t[..., b] = y[..., a] + y[..., b]
    return t


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,hq,hk,dh,rot,inter,far", [
    (1, 1, 1, 16, 16, False, False), (37, 4, 4, 32, 32, False, True), (130, 3, 1, 64, 32, False, False),
    (65, 8, 2, 128, 128, True, True), (33, 4, 4, 16, 16, True, True), (50, 2, 2, 32, 0, False, False),
    (77, 5, 3, 64, 16, True, False), (9, 64, 64, 16, 16, False, False), (4000, 2, 2, 32, 16, False, True)])
def test_qkrot_forward_and_backward(dt, n, hq, hk, dh, rot, inter, far):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    rng, q, k, gq, gk, pos = rot_problem(dt, n, hq, hk, dh, n + dh, far)
    p = hg.QkRotParams(dev(gq, td), dev(gk, td), hq, hk, rot=rot, base=1000.0, eps=1e-4, interleaved=inter)
    Q, K, P = strided(q, td), strided(k, td), dev(pos)
    qo, ko = nans((n, hq, dh), td), nans((n, hk, dh), td)
    hg.hg_qkrot_fwd(p, Q, K, P, qo, ko)
    how = (rot, 1000.0, 1e-4, inter)
    for got, x, g, name in ((qo, q, gq, "q"), (ko, k, gk, "k")):
        near(got, OH.qkrot_forward(f64(x), f64(g), pos, *how), rot_terms(None, f64(x), f64(g), pos, *how), rot_rel(dt),
             name)
    dyq, dyk = draw(rng, dt, n, hq, dh), draw(rng, dt, n, hk, dh)
    dq, dk = nans((n, hq, dh), td), nans((n, hk, dh), td)
    grads = {"gamma_q": nans((dh,), torch.float32), "gamma_k": nans((dh,), torch.float32)}
    scratch = torch.empty(hg.hg_qkrot_workspace_size(p, n), dtype=torch.uint8, device="cuda")
    hg.hg_qkrot_bwd(p, Q, K, P, strided(dyq, td), strided(dyk, td), dq, dk, grads, scratch)
    for got, ggot, x, g, dy, name in ((dq, grads["gamma_q"], q, gq, dyq, "dq"), (dk, grads["gamma_k"], k, gk, dyk, "dk")):
        x, g, dy = f64(x), f64(g), f64(dy)
        want, dg = OH.qkrot_backward(x, g, pos, *how, dy)
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + how[2])
        u = np.abs(x) * r
        a, b = OH.pair_index(rot, inter)
        t = np.abs(dy).copy()
        t[..., a] = t[..., b] = np.abs(dy)[..., a] + np.abs(dy)[..., b]
        c = t * np.abs(g)
        near(got, want, r * (c + u * (c * u).mean(-1, keepdims=True)), (U[dt], 2 * rot_rel(dt)[1]), name)
        # a sum over the rows of a head: at most n heads terms, in runs of at most n
        near(ggot, dg, (t * u).sum((0, 1)), (0, rot_rel(dt)[1] + n * x.shape[1] * F32), name + " gain")


def test_qkrot_in_place_default_positions_and_no_keys():
    need_gpu()
    hg = lib()
    _, q, k, gq, gk, _ = rot_problem("bf16", 70, 4, 2, 32, 5, False)
    td = torch.bfloat16
    p = hg.QkRotParams(dev(gq, td), dev(gk, td), 4, 2)
    a, b = nans((70, 4, 32), td), nans((70, 2, 32), td)
    hg.hg_qkrot_fwd(p, dev(q, td), dev(k, td), dev(np.arange(70)), a, b)
    Q, K = dev(q, td), dev(k, td)
    hg.hg_qkrot_fwd(p, Q, K, None, Q, K)
    assert torch.equal(Q, a) and torch.equal(K, b)
    alone = hg.QkRotParams(dev(gq, td), None, 4, 0)
    c = nans((70, 4, 32), td)
    hg.hg_qkrot_fwd(alone, dev(q, td), None, None, c, None)
    assert torch.equal(c, a)
    plain = hg.QkRotParams(None, None, 4, 2, d_h=32, dtype=td)  # no gains: ones
    ones = hg.QkRotParams(torch.ones(32, dtype=td, device="cuda"), torch.ones(32, dtype=td, device="cuda"), 4, 2)
    x, y = [nans((70, 4, 32), td) for _ in range(2)], [nans((70, 2, 32), td) for _ in range(2)]
    for prm, xo, yo in zip((plain, ones), x, y):
        hg.hg_qkrot_fwd(prm, dev(q, td), dev(k, td), None, xo, yo)
    assert torch.equal(*x) and torch.equal(*y)
    # upstream gradients overwritten in place; a gain's gradient left out
    scratch = torch.empty(hg.hg_qkrot_workspace_size(p, 70), dtype=torch.uint8, device="cuda")
    g1 = {"gamma_q": nans((32,), torch.float32), "gamma_k": nans((32,), torch.float32)}
    dq, dk = nans((70, 4, 32), td), nans((70, 2, 32), td)
    up = dev(k, td)
    hg.hg_qkrot_bwd(p, dev(q, td), dev(k, td), None, a, up, dq, dk, g1, scratch)
    g2 = {"gamma_k": nans((32,), torch.float32)}
    da, db = a.clone(), up.clone()
    hg.hg_qkrot_bwd(p, dev(q, td), dev(k, td), None, da, db, da, db, g2, scratch)
    assert torch.equal(da, dq) and torch.equal(db, dk) and torch.equal(g2["gamma_k"], g1["gamma_k"])


def test_qkrot_a_row_keeps_its_own_troubles():
    """Infinities, NaN and zero rows stay in their row; an empty call writes zero gain gradients."""
    need_gpu()
    hg = lib()
    _, q, k, gq, gk, pos = rot_problem("f32", 40, 2, 2, 32, 6, False)
    p = hg.QkRotParams(dev(gq), dev(gk), 2, 2)
    ref = [nans((40, 2, 32), torch.float32) for _ in range(2)]
    hg.hg_qkrot_fwd(p, dev(q), dev(k), dev(pos), *ref)
    q2 = q.copy()
    q2[3], q2[7, 1], q2[9] = np.nan, np.inf, 0
    out = [nans((40, 2, 32), torch.float32) for _ in range(2)]
    hg.hg_qkrot_fwd(p, dev(q2), dev(k), dev(pos), *out)
    keep = torch.ones(40, 2, dtype=torch.bool, device="cuda")
    keep[3] = keep[7, 1] = keep[9] = False
    assert torch.equal(out[0][keep], ref[0][keep]) and torch.equal(out[1], ref[1])
    assert (out[0][9] == 0).all()
    g = {x: nans((32,), torch.float32) for x in ("gamma_q", "gamma_k")}
    e = torch.empty(0, 2, 32, device="cuda")
    hg.hg_qkrot_fwd(p, e, e, None, e, e)
    hg.hg_qkrot_bwd(p, e, e, None, e, e, e, e, g, None)
    assert (g["gamma_q"] == 0).all() and (g["gamma_k"] == 0).all()


# ------------------------------------------------------------------------------------------------- decay
LD = np.array([-0.01, -0.7, 0.0, -6.0, -1e-4, -150.0, -0.05, -0.3], np.float32)


def decay_problem(dt, n, T, h, dh, seed, ragged, state):
    rng = np.random.default_rng(seed)
    q, k, v, do = (draw(rng, dt, n, T, h, dh) for _ in range(4))
    lens = None
    if ragged:
        lens = rng.integers(0, T + 1, n).astype(np.int32)
        lens[0], lens[-1] = 0, T
    S = rng.standard_normal((2, n, h, dh, dh)).astype(np.float32) if state else (None, None)
    return q, k, v, do, lens, S[0], S[1]


def past(x, lens):
    """x with NaN where a sequence has ended."""
    if lens is not None:
        x = x.copy()
        x[np.arange(x.shape[1])[None] >= lens[:, None]] = np.nan
    return x


# Rows: bf16 rounds the weights of a chunk (the products q k of its positions times their decay) and the state that
# enters it once each: r = 2 u.  States are fp32 sums of terms in 24 bits; 2^-15 is allowed here, and
# test_gpu_history_edges.py has the bound of such sums.
# e: sums of at most T d_h terms in chunks (T + 2 d_h), decays exp(x) with |x| <= 5 + rounding 2^-22, 4 of them.
def decay_rel(dt, T, dh, out):
    e = (T + 2 * dh + 80) * F32
    if dt == "f32":
        return (U["f32"] if out == "rows" else 0, e)
    return (U["bf16"], 2 * U["bf16"] + e) if out == "rows" else (0, 2.0**-15 + e)


CASES = [(1, 1, 1, 16, False, False), (3, 1, 2, 32, True, True), (2, 15, 3, 32, True, False), (5, 16, 4, 16, False, True),
         (4, 17, 2, 64, True, True), (3, 33, 1, 128, True, True), (2, 100, 5, 16, True, True), (2, 70, 2, 64, False, False),
         (1, 200, 4, 32, False, True), (70, 5, 8, 16, True, False), (1, 700, 1, 32, False, True),
         (2, 1100, 2, 64, True, True), (1, 530, 1, 128, True, True)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,h,dh,ragged,state", CASES)
def test_decay_forward_and_backward(dt, n, T, h, dh, ragged, state):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    q, k, v, do, lens, S, dS = decay_problem(dt, n, T, h, dh, n + T + dh, ragged, state)
    ld, c = LD[:h], dh ** -0.5
    p = hg.DecayParams(dev(ld), dh, td, scale=c)
    fw, bw = hg.hg_decay_workspace_size(p, n, T)
    work = torch.empty(max(fw, bw), dtype=torch.uint8, device="cuda")
    Q, K, V, DO = (strided(past(x, lens), td) for x in (q, k, v, do))
    L, S0, DS = (None if x is None else dev(x) for x in (lens, S, dS))
    o, last = nans((n, T, h, dh), td), nans((n, h, dh, dh), torch.float32)
    hg.hg_decay_fwd(p, Q, K, V, L, S0, o, last, work)
    args = [f64(x) for x in (q, k, v)] + [f64(ld), np.float64(np.float32(c))]
    want = OH.decay_forward(*args, lens, f64(S))
    terms = OH.decay_forward(*args, lens, f64(S), magnitude=True)
    for got, w, t, name in ((o, want[0], terms[0], "rows"), (last, want[1], terms[1], "state")):
        near(got, w, t, decay_rel(dt, T, dh, name), name)
    grads = [nans((n, T, h, dh), td) for _ in range(3)] + [nans((n, h, dh, dh), torch.float32)]
    hg.hg_decay_bwd(p, Q, K, V, L, S0, DO, DS, *grads, work)
    want = OH.decay_backward(*args, f64(do), lens, f64(S), f64(dS))
    terms = OH.decay_backward(*args, f64(do), lens, f64(S), f64(dS), magnitude=True)
    for got, w, t, name in zip(grads, want, terms, ("dq", "dk", "dv", "state")):
        near(got, w, t, decay_rel(dt, T, dh, "state" if name == "state" else "rows"), name)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_decay_layouts_and_states_in_place(dt):
    """Sequences nested in positions (T x n), lens outside [0, T], states updated in place, nothing asked for."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    n, T, h, dh = 6, 21, 2, 32
    q, k, v, do, lens, S, dS = decay_problem(dt, n, T, h, dh, 9, True, True)
    p = hg.DecayParams(dev(LD[:h]), dh, td)
    a, last = nans((n, T, h, dh), td), nans((n, h, dh, dh), torch.float32)
    hg.hg_decay_fwd(p, *(dev(x, td) for x in (q, k, v)), dev(lens), dev(S), a, last, None)
    flip = lambda x: dev(np.ascontiguousarray(x.swapaxes(0, 1)), td).transpose(0, 1)  # noqa: E731
    b = nans((T, n, h, dh), td).transpose(0, 1)
    state = dev(S)
    hg.hg_decay_fwd(p, flip(q), flip(k), flip(v), dev(lens), state, b, state, None)
    assert torch.equal(a, b) and torch.equal(last, state)
    odd = lens.copy()
    odd[lens == 0] = -5
    odd[lens == T] = T + 9
    c = nans((n, T, h, dh), td)
    hg.hg_decay_fwd(p, *(dev(x, td) for x in (q, k, v)), dev(odd), dev(S), c, None, None)
    assert torch.equal(a, c)
    g1 = [nans((n, T, h, dh), td) for _ in range(3)] + [nans((n, h, dh, dh), torch.float32)]
    g2 = [nans((T, n, h, dh), td).transpose(0, 1) for _ in range(3)] + [dev(dS)]
    x = [dev(y, td) for y in (q, k, v)]
    hg.hg_decay_bwd(p, *x, dev(lens), dev(S), dev(do, td), dev(dS), *g1, None)
    hg.hg_decay_bwd(p, flip(q), flip(k), flip(v), dev(lens), dev(S), flip(do), g2[3], *g2, None)
    assert all(torch.equal(y, z) for y, z in zip(g1, g2))
    # no positions, no sequences
    e = torch.empty(n, 0, h, dh, dtype=td, device="cuda")
    hg.hg_decay_fwd(p, e, e, e, None, dev(S), e, last, None)
    assert torch.equal(last, dev(S))
    hg.hg_decay_fwd(p, e, e, e, None, None, e, last, None)
    assert (last == 0).all()
    z = torch.empty(0, T, h, dh, dtype=td, device="cuda")
    hg.hg_decay_fwd(p, z, z, z, None, None, z, None, None)


# Each warp takes several heads here (an SM holds 8 to 20 warps): the order in which they follow one another, dealt out
# (carries past the last sequence and the last scan) and claimed.
@pytest.mark.parametrize("n,T,h,dh,ragged", [(1201, 19, 8, 16, True), (997, 35, 5, 32, True), (1300, 3, 7, 32, False),
                                             (1003, 18, 3, 64, True), (331, 17, 4, 128, True), (1100, 130, 3, 32, True),
                                             (450, 130, 4, 64, True)])
def test_decay_of_many_histories(n, T, h, dh, ragged):
    """The same bits as those of the histories in small batches, in which a warp has one head."""
    need_gpu()
    hg = lib()
    td = torch.bfloat16
    q, k, v, do, lens, S, dS = decay_problem("bf16", n, T, h, dh, n, ragged, True)
    if lens is not None:
        lens[5:9] = 0
        lens[-3:] = 0
    p = hg.DecayParams(dev(LD[:h]), dh, td, scale=dh ** -0.5)
    Q, K, V, DO = (strided(past(x, lens), td) for x in (q, k, v, do))
    L, S0, DS = (None if x is None else dev(x) for x in (lens, S, dS))

    def run(at):
        some = [None if x is None else x[at] for x in (Q, K, V, L, S0, DO, DS)]
        m = some[0].shape[0]
        work = torch.empty(max(hg.hg_decay_workspace_size(p, m, T)), dtype=torch.uint8, device="cuda")
        out = [nans((m, T, h, dh), td) for _ in range(4)] + [nans((m, h, dh, dh), torch.float32) for _ in range(2)]
        hg.hg_decay_fwd(p, *some[:5], out[0], out[4], work)
        hg.hg_decay_bwd(p, *some[:5], some[5], some[6], *out[1:4], out[5], work)
        return out

    whole = run(slice(None))
    parts = [run(slice(i, i + 50)) for i in range(0, n, 50)]
    for x, y in zip(whole, (torch.cat(z) for z in zip(*parts))):
        assert torch.isfinite(x).all() and torch.equal(x, y)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,dh", [(3, 1300, 64), (5, 300, 128), (2, 2100, 16)])
def test_decay_state_gradient_in_place_of_a_long_history(dt, n, T, dh):
    """dS_in in the place of dS_out, which the gradient of the keys reads too: segments, claimed lengths."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    q, k, v, do, lens, S, dS = decay_problem(dt, n, T, 2, dh, T, True, True)
    p = hg.DecayParams(dev(LD[:2]), dh, td, scale=0.25)
    x = [dev(y, td) for y in (q, k, v)]
    work = torch.empty(hg.hg_decay_workspace_size(p, n, T)[1], dtype=torch.uint8, device="cuda")
    runs = []
    for state, out in ((dev(dS), nans((n, 2, dh, dh), torch.float32)), (dev(dS), None)):
        g = [nans((n, T, 2, dh), td) for _ in range(3)] + [state if out is None else out]
        hg.hg_decay_bwd(p, *x, dev(lens), dev(S), dev(do, td), state, *g, work)
        runs.append(g)
    assert all(torch.equal(y, z) for y, z in zip(*runs))
    with pytest.raises(hg.HGError, match="S_in"):
        hg.hg_decay_bwd(p, *x, dev(lens), runs[0][3], dev(do, td), None, *runs[0], work)


def test_decay_long_memory_keeps_its_decay():
    """gamma close to 1 over thousands of positions: keys that are zero after the first leave gamma^t q k v alone."""
    need_gpu()
    hg = lib()
    T, dh, ld = 6000, 32, np.array([-2.0**-12], np.float32)
    x = np.zeros((1, T, 1, dh), np.float32)
    x[0, 0] = 1
    one = np.ones((1, T, 1, dh), np.float32)
    for dt in ("f32", "bf16"):
        td = tdtype(dt)
        p = hg.DecayParams(dev(ld), dh, td)
        work = torch.empty(hg.hg_decay_workspace_size(p, 1, T)[0], dtype=torch.uint8, device="cuda")
        o, last = nans((1, T, 1, dh), td), nans((1, 1, dh, dh), torch.float32)
        hg.hg_decay_fwd(p, dev(one, td), dev(x, td), dev(x, td), None, None, o, last, work)
        want = dh * np.exp(np.float64(ld[0]) * np.arange(T))[None, :, None, None] * np.ones((1, T, 1, dh))
        # a frame's move rounds the state once, 2^-22 with its exp, at most once in 5 / 2^-12 positions or a segment
        near(o, want, want, (U[dt], 40 * F32 + (U[dt] if dt == "bf16" else 0)), "rows")
        near(last, want[0, -1, 0, 0] / dh * np.ones((1, 1, dh, dh)), np.ones((1, 1, dh, dh)),
             (0, 40 * F32 + (2.0**-16 if dt == "bf16" else 0)), "state")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,dh", [(1, 1, 16), (19, 3, 32), (40, 2, 64), (7, 5, 128)])
def test_decay_step(dt, n, h, dh):
    """One snapshot from a carried state, against the recurrence; rows without one keep their state."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    q, k, v, _, _, S, _ = decay_problem(dt, n, 1, h, dh, n + dh, False, True)
    live = (np.random.default_rng(n).random(n) < 0.6).astype(np.int32)
    live[0] = 1
    p = hg.DecayParams(dev(LD[:h]), dh, td, scale=0.5)
    o, out = nans((n, h, dh), td), nans((n, h, dh, dh), torch.float32)
    Q, K, V = (strided(x[:, 0], td) for x in (q, k, v))
    hg.hg_decay_step(p, Q, K, V, dev(live), dev(S), o, out)
    args = [f64(x) for x in (q, k, v)] + [f64(LD[:h]), 0.5]
    want = OH.decay_forward(*args, live, f64(S))
    terms = OH.decay_forward(*args, live, f64(S), magnitude=True)
    near(o, want[0][:, 0], terms[0][:, 0], (U[dt], (dh + 40) * F32), "row")
    near(out, want[1], terms[1], (0, 8 * F32), "state")
    state, o2 = dev(S), nans((n, h, dh), td)
    hg.hg_decay_step(p, Q, K, V, dev(live), state, o2)
    assert torch.equal(state, out) and torch.equal(o2, o)
    assert torch.equal(out[dev(live) == 0], dev(S)[dev(live) == 0])
    hg.hg_decay_step(p, Q, K, V, None, dev(S), o2, out)
    want = OH.decay_forward(*args, None, f64(S))
    near(out, want[1], OH.decay_forward(*args, None, f64(S), magnitude=True)[1], (0, 8 * F32), "all live")
    e, es = torch.empty(0, h, dh, dtype=td, device="cuda"), torch.empty(0, h, dh, dh, device="cuda")
    hg.hg_decay_step(p, e, e, e, None, es, e)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_steps_follow_the_scan(dt):
    """A history taken at once leaves the state that its snapshots leave one by one."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    n, T, h, dh = 5, 23, 4, 32
    q, k, v, *_ = decay_problem(dt, n, T, h, dh, 1, False, False)
    p = hg.DecayParams(dev(LD[:h]), dh, td)
    Q, K, V = (dev(x, td) for x in (q, k, v))
    o, last = nans((n, T, h, dh), td), nans((n, h, dh, dh), torch.float32)
    hg.hg_decay_fwd(p, Q, K, V, None, None, o, last, None)
    state, row = torch.zeros(n, h, dh, dh, device="cuda"), nans((n, T, h, dh), td)
    for t in range(T):
        hg.hg_decay_step(p, Q[:, t], K[:, t], V[:, t], None, state, row[:, t])
    args = [f64(x) for x in (q, k, v)] + [f64(LD[:h]), 1.0]
    want, terms = OH.decay_forward(*args), OH.decay_forward(*args, magnitude=True)
    for got, name in ((o, "scan"), (row, "steps")):
        near(got, want[0], terms[0], decay_rel(dt, 4 * T, dh, "rows"), name)
    for got, name in ((last, "scan"), (state, "steps")):
        near(got, want[1], terms[1], decay_rel(dt, 4 * T, dh, "state"), name)


# ------------------------------------------------------------------------------------------------ gated block
def ffn_problem(dt, n, d, f, seed):
    rng = np.random.default_rng(seed)
    a = np.sqrt(2 / (d + f))
    return [draw(rng, dt, n, d), draw(rng, dt, d, f, scale=a), draw(rng, dt, d, f, scale=a),
            draw(rng, dt, f, d, scale=a), draw(rng, dt, n, d)]


def ffn_check(hg, dt, n, d, f, act, res):
    td = tdtype(dt)
    X, Wg, Wu, Wd, dY = ffn_problem(dt, n, d, f, n + d + f)
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)), act=act, residual=res)
    fw, bw = hg.hg_ffn_workspace_size(p, n)
    work = torch.empty(max(fw, bw), dtype=torch.uint8, device="cuda")
    Xd, dYd, Y, dX = dev(X, td), dev(dY, td), nans((n, d), td), nans((n, d), td)
    hg.hg_ffn_fwd(p, Xd, Y, work)
    X, Wg, Wu, Wd, dY = (f64(x) for x in (X, Wg, Wu, Wd, dY))
    G, U_ = X @ Wg, X @ Wu
    aG, aU = np.abs(X) @ np.abs(Wg), np.abs(X) @ np.abs(Wu)
    A, dA = OH.act(G, act)
    # fp32: the projections within d 2^-24 of aG, aU; |act(x)| <= |x|, |act'| <= 1.13, act and act' change by at most
    # 1.13 and 0.6 (GELU: 1.2) per unit; the gates' functions 30 steps.  bf16: the hidden row rounded once.
    e = 3 * (d + f + 40) * F32
    r = U["bf16"] if dt == "bf16" else 0
    y = OH.ffn_forward(X, Wg, Wu, Wd, act, res)
    t = (aG * aU) @ np.abs(Wd) + (np.abs(X) if res else 0)
    near(Y, y, (r * (np.abs(A * U_) @ np.abs(Wd)) + e * t) / max(r + e, 1e-30), (U[dt], r + e), "Y")
    g = {"W_gate": nans((d, f), torch.float32), "W_up": nans((d, f), torch.float32), "W_down": nans((f, d), torch.float32)}
    hg.hg_ffn_bwd(p, Xd, dYd, dX, g, work)
    want = OH.ffn_backward(X, Wg, Wu, Wd, act, res, dY)
    dH, adH = dY @ Wd.T, np.abs(dY) @ np.abs(Wd.T)
    dG, dU = dH * U_ * dA, dH * A
    tG, tU, tH = adH * aU * (1.2 + 1.2 * aG), adH * aG * 1.2, aG * aU * 1.2
    # bf16: dG and dU rounded once for dX; for the weights, whose sums are fp32, each of dG, dU and H as a sum of two
    # bf16 numbers (2^-16)
    s = 2.0**-16 if dt == "bf16" else 0
    terms = r * (np.abs(dG) @ np.abs(Wg.T) + np.abs(dU) @ np.abs(Wu.T)) + e * (tG @ np.abs(Wg.T) + tU @ np.abs(Wu.T) + np.abs(dY))
    near(dX, want[0], terms, (U[dt], 1.0), "dX")
    e += n * F32
    for key, w, left, right, tr in (("W_gate", want[1], X, dG, tG), ("W_up", want[2], X, dU, tU)):
        near(g[key], w, s * (np.abs(left.T) @ np.abs(right)) + e * (np.abs(left.T) @ tr), (0, 1.0), key)
    near(g["W_down"], want[3], s * (np.abs(A * U_).T @ np.abs(dY)) + e * (tH.T @ np.abs(dY)), (0, 1.0), "W_down")
    return p, Xd, dYd, Y, dX, g, work


FFN = [(1, 64, 8, "silu", False), (127, 64, 200, "gelu_tanh", True), (128, 128, 64, "silu", True),
       (129, 128, 384, "silu", False), (300, 256, 136, "relu", True), (257, 256, 704, "silu", True),
       (500, 128, 72, "none", False), (1000, 64, 264, "silu", True)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,f,act,res", FFN)
def test_ffn_forward_and_backward(dt, n, d, f, act, res):
    need_gpu()
    hg = lib()
    p, X, dY, Y, dX, g, work = ffn_check(hg, dt, n, d, f, act, res)
    # parts left out give the same others
    alone = torch.empty_like(dX)
    hg.hg_ffn_bwd(p, X, dY, alone, None, work)
    assert torch.equal(alone, dX)
    again = {k: nans(v.shape, torch.float32) for k, v in g.items()}
    hg.hg_ffn_bwd(p, X, dY, None, again, work)
    assert all(torch.equal(again[k], g[k]) for k in g)


@pytest.mark.parametrize("dt,d,f", [("f32", 64, 40), ("bf16", 64, 40), ("bf16", 64, 200), ("bf16", 128, 136),
                                    ("bf16", 128, 256), ("bf16", 256, 72), ("bf16", 256, 320)])
def test_ffn_many_row_tiles(dt, d, f):
    """More row tiles than CTAs, with one to five chunks of hidden features: every tile is taken, none twice, and a
    row's values do not depend on the tiles around it, whatever turn their chunks take."""
    need_gpu()
    hg = lib()
    n = 45_001
    td = tdtype(dt)
    X, Wg, Wu, Wd, dY = ffn_problem(dt, 129, d, f, 3)
    at = torch.arange(n, device="cuda") % 129
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)))
    work = torch.empty(max(hg.hg_ffn_workspace_size(p, n)), dtype=torch.uint8, device="cuda")
    few, many = nans((129, d), td), nans((n, d), td)
    hg.hg_ffn_fwd(p, dev(X, td), few, work)
    big, up = dev(X, td)[at].contiguous(), dev(dY, td)[at].contiguous()
    hg.hg_ffn_fwd(p, big, many, work)
    assert torch.equal(many, few[at])
    g = {"W_gate": nans((d, f), torch.float32), "W_up": nans((d, f), torch.float32), "W_down": nans((f, d), torch.float32)}
    hg.hg_ffn_bwd(p, dev(X, td), dev(dY, td), few, None, work)
    hg.hg_ffn_bwd(p, big, up, many, g, work)
    assert torch.equal(many, few[at])
    X, Wg, Wu, Wd, dY = (f64(x) for x in (X, Wg, Wu, Wd, dY))
    times = np.bincount(host(at).astype(int), minlength=129)[:, None]
    want = OH.ffn_backward(X, Wg, Wu, Wd, "silu", False, dY * times)
    for key, w in zip(("W_gate", "W_up", "W_down"), want[1:]):
        # 349 equal rows of 129: relative to the whole, the sums' order (45001 2^-24) and the split of 2^-16
        assert np.abs(host(g[key]) - w).max() <= 3e-3 * np.abs(w).max(), key
        assert np.linalg.norm(host(g[key]) - w) <= 1e-4 * np.linalg.norm(w), key


@pytest.mark.parametrize("d,f", [(64, 40), (64, 136), (128, 72), (128, 200), (256, 64), (256, 264)])
def test_ffn_many_row_tiles_with_a_residual(d, f):
    """Y starts at X and dX at dY, whose places take the next tile early: rows of several tiles a CTA as those of one."""
    need_gpu()
    hg = lib()
    n, m = 60_003, 331
    td = torch.bfloat16
    X, Wg, Wu, Wd, dY = ffn_problem("bf16", m, d, f, 7)
    at = torch.arange(n, device="cuda") % m
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)), act="gelu_tanh", residual=True)
    work = torch.empty(max(hg.hg_ffn_workspace_size(p, n)), dtype=torch.uint8, device="cuda")
    few, many = nans((m, d), td), nans((n, d), td)
    hg.hg_ffn_fwd(p, dev(X, td), few, None)
    big, up = dev(X, td)[at].contiguous(), dev(dY, td)[at].contiguous()
    hg.hg_ffn_fwd(p, big, many, None)
    assert torch.equal(many, few[at])
    hg.hg_ffn_bwd(p, dev(X, td), dev(dY, td), few, None, work)
    hg.hg_ffn_bwd(p, big, up, many, None, work)
    assert torch.equal(many, few[at])


def far(x, stride):
    """The rows of x, whose first index lies `stride` values apart."""
    t = torch.empty(stride * (x.shape[0] - 1) + x[0].numel(), dtype=x.dtype, device="cuda")
    v = t.as_strided(x.shape, (stride, *x.stride()[1:]))
    v.copy_(x)
    return v


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_offsets_past_32_bits_and_shared_rows(dt):
    """Rows 2^31 values apart give the bits of rows side by side; so do inputs whose rows are one row (stride 0)."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    n, T, h, dh, step = 2, 19, 2, 32, (1 << 31) + 64
    rng = np.random.default_rng(1)
    x = [dev(draw(rng, dt, n, T, h, dh), td) for _ in range(4)]
    p = hg.DecayParams(dev(LD[:h]), dh, td)
    o = nans((n, T, h, dh), td)
    hg.hg_decay_fwd(p, *x[:3], None, None, o, None, None)
    g = [nans((n, T, h, dh), td) for _ in range(3)]
    hg.hg_decay_bwd(p, *x[:3], None, None, x[3], None, *g, None, None)
    fo = far(nans((n, T, h, dh), td), step)
    fq, fk = far(x[0], step), far(x[1], step)
    hg.hg_decay_fwd(p, fq, fk, x[2], None, None, fo, None, None)
    assert torch.equal(fo, o)
    fo.fill_(float("nan"))
    hg.hg_decay_bwd(p, fq, fk, x[2], None, None, x[3], None, g[0].clone(), fo, g[2].clone(), None, None)
    assert torch.equal(fo, g[1])
    r = hg.QkRotParams(None, None, h, h, d_h=dh, dtype=td)
    a, b = nans((n, h, dh), td), nans((n, h, dh), td)
    hg.hg_qkrot_fwd(r, x[0][:, 1], x[1][:, 2], None, a, b)
    hg.hg_qkrot_fwd(r, fq[:, 1], fk[:, 2], None, fo[:, 0], fo[:, 1])
    assert torch.equal(fo[:, 0], a) and torch.equal(fo[:, 1], b)
    del fq, fk, fo
    one = x[0][:1, :1].expand(n, T, h, dh)
    hg.hg_decay_fwd(p, one, one, x[2], None, None, o, None, None)
    o2 = nans((n, T, h, dh), td)
    hg.hg_decay_fwd(p, one.contiguous(), one.contiguous(), x[2], None, None, o2, None, None)
    assert torch.equal(o, o2)
    hg.hg_qkrot_fwd(r, one[:, 0], x[1][:, 2], None, a, b)
    assert torch.equal(a[0], hg_rot(hg, r, x[0][:1, 0], h, dh, td)[0])


def hg_rot(hg, r, q, h, dh, td):
    a, b = nans((1, h, dh), td), nans((1, h, dh), td)
    hg.hg_qkrot_fwd(r, q, q.clone(), None, a, b)
    return a


def test_states_past_32_bits():
    """A step whose states hold more than 2^31 values: the last nodes' are those of a step on them alone."""
    need_gpu()
    hg = lib()
    n, h, dh = 530_001, 4, 32
    p = hg.DecayParams(dev(LD[:h]), dh, torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(n, h, dh, device="cuda", generator=gen, dtype=torch.bfloat16) for _ in range(3))
    S = torch.full((n, h, dh, dh), 0.5, device="cuda")
    assert S.numel() > 1 << 31
    o = nans((n, h, dh), torch.bfloat16)
    hg.hg_decay_step(p, q, k, v, None, S, o)
    few = torch.full((7, h, dh, dh), 0.5, device="cuda")
    o2 = nans((7, h, dh), torch.bfloat16)
    hg.hg_decay_step(p, q[-7:], k[-7:], v[-7:], None, few, o2)
    assert torch.equal(S[-7:], few) and torch.equal(o[-7:], o2)
    want = nans((7, 1, h, dh), torch.bfloat16)
    S[-7:] = 0.5
    hg.hg_decay_fwd(p, q[-7:, None], k[-7:, None], v[-7:, None], None, S[-7:], want, S[-7:], None)
    # terms: the decayed 0.5 and products below 25 (two normal numbers of five deviations)
    near(S[-7:], host(few), np.abs(host(few)) + 25, decay_rel("bf16", 1, dh, "state"), "scan of one")


def test_ffn_empty():
    need_gpu()
    hg = lib()
    _, Wg, Wu, Wd, _ = ffn_problem("bf16", 1, 64, 16, 0)
    td = torch.bfloat16
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)))
    e = torch.empty(0, 64, dtype=td, device="cuda")
    g = {"W_gate": nans((64, 16), torch.float32), "W_up": nans((64, 16), torch.float32), "W_down": nans((16, 64), torch.float32)}
    hg.hg_ffn_fwd(p, e, e, None)
    hg.hg_ffn_bwd(p, e, e, e, g, None)
    assert all((x == 0).all() for x in g.values())


# ------------------------------------------------------------------------------------------------- together
class Encoder:
    """Norm and rotation, the scan over the history, the gated block on its rows, and back."""

    def __init__(self, hg, dt, n, T, h, dh, f, seed):
        self.hg, self.td, self.n, self.T, self.h, self.dh, self.d = hg, tdtype(dt), n, T, h, dh, h * dh
        rng = np.random.default_rng(seed)
        self.host = {"qkv": draw(rng, dt, n, T, 3, h, dh), "gain": 1 + draw(rng, dt, 2, dh, scale=0.125),
                     "dY": draw(rng, dt, n * T, self.d), "pos": rng.integers(0, 1000, (n, T)),
                     "lens": rng.integers(0, T + 1, n).astype(np.int32)}
        if dt == "bf16":
            self.host["gain"] = bf16_round(self.host["gain"])
        self.w = ffn_problem(dt, 1, self.d, f, seed)[1:4]
        td, c = self.td, torch.cuda.current_stream()
        self.rot = hg.QkRotParams(*(dev(x, td) for x in self.host["gain"]), h, h)
        self.dec = hg.DecayParams(dev(LD[:h]), dh, td, scale=0.25)
        self.ffn = hg.FfnParams(*(dev(x, td) for x in self.w), residual=True)
        self.t = {k: dev(self.host[k], td) for k in ("qkv", "dY")}
        self.t["pos"], self.t["lens"] = dev(self.host["pos"].reshape(-1)), dev(self.host["lens"])
        new = lambda *s, dtype=td: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.q, self.k, self.dq, self.dk, self.dv = (new(n, T, h, dh) for _ in range(5))
        self.o, self.y, self.do = new(n, T, h, dh), new(n * T, self.d), new(n * T, self.d)
        self.S, self.dS = new(n, h, dh, dh, dtype=f32), new(n, h, dh, dh, dtype=f32)
        self.g = {"gamma_q": new(dh, dtype=f32), "gamma_k": new(dh, dtype=f32), "W_gate": new(self.d, f, dtype=f32),
                  "W_up": new(self.d, f, dtype=f32), "W_down": new(f, self.d, dtype=f32)}
        need = max(*hg.hg_decay_workspace_size(self.dec, n, T), *hg.hg_ffn_workspace_size(self.ffn, n * T),
                   hg.hg_qkrot_workspace_size(self.rot, n * T))
        self.work = torch.empty(need, dtype=torch.uint8, device="cuda")
        c.synchronize()

    def run(self, stream=None):
        hg, t, rows = self.hg, self.t, self.n * self.T
        x = t["qkv"].view(rows, 3, self.h, self.dh)
        v = t["qkv"][:, :, 2]
        flat = lambda z: z.view(rows, self.h, self.dh)  # noqa: E731
        hg.hg_qkrot_fwd(self.rot, x[:, 0], x[:, 1], t["pos"], flat(self.q), flat(self.k), stream=stream)
        hg.hg_decay_fwd(self.dec, self.q, self.k, v, t["lens"], None, self.o, self.S, self.work, stream=stream)
        hg.hg_ffn_fwd(self.ffn, self.o.view(rows, self.d), self.y, self.work, stream=stream)
        hg.hg_ffn_bwd(self.ffn, self.o.view(rows, self.d), t["dY"], self.do, self.g, self.work, stream=stream)
        hg.hg_decay_bwd(self.dec, self.q, self.k, v, t["lens"], None, self.do.view_as(self.o), None, self.dq, self.dk,
                        self.dv, self.dS, self.work, stream=stream)
        hg.hg_qkrot_bwd(self.rot, x[:, 0], x[:, 1], t["pos"], flat(self.dq), flat(self.dk), flat(self.dq),
                        flat(self.dk), self.g, self.work, stream=stream)

    def outputs(self):
        return {"y": self.y, "S": self.S, "dq": self.dq, "dk": self.dk, "dv": self.dv, "dS": self.dS, **self.g}

    def oracle(self):
        a = {k: f64(x) for k, x in self.host.items()}
        n, T, rows = self.n, self.T, self.n * self.T
        how = (self.dh, 10000.0, 1e-6, False)
        pos, lens = self.host["pos"].reshape(-1), self.host["lens"]
        flat = lambda z: z.reshape(rows, self.h, self.dh)  # noqa: E731
        q0, k0, v = (a["qkv"][:, :, i] for i in range(3))
        q, k = (OH.qkrot_forward(flat(x), g, pos, *how).reshape(q0.shape) for x, g in ((q0, a["gain"][0]), (k0, a["gain"][1])))
        args = (q, k, v, f64(LD[:self.h]), 0.25)
        o, S = OH.decay_forward(*args, lens)
        w = [f64(x) for x in self.w]
        o2 = o.reshape(rows, self.d)
        y = OH.ffn_forward(o2, *w, "silu", True)
        do, wg, wu, wd = OH.ffn_backward(o2, *w, "silu", True, a["dY"])
        dq, dk, dv, dS = OH.decay_backward(*args, do.reshape(o.shape), lens)
        dq, gq = OH.qkrot_backward(flat(q0), a["gain"][0], pos, *how, flat(dq))
        dk, gk = OH.qkrot_backward(flat(k0), a["gain"][1], pos, *how, flat(dk))
        return {"y": y, "S": S, "dq": dq.reshape(q0.shape), "dk": dk.reshape(q0.shape), "dv": dv, "dS": dS, "gamma_q": gq,
                "gamma_k": gk, "W_gate": wg, "W_up": wu, "W_down": wd}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_encoder_forward_and_backward(dt):
    """The operators one after another, rows behind a sequence's end among them (zero rows of the block's input).
    Normwise: each of the five stages rounds once or twice, relative to the norm 2^-8 each in bf16 (their errors add
    like independent ones; 10 steps are allowed), and sums some hundred terms in fp32."""
    need_gpu()
    e = Encoder(lib(), dt, 6, 40, 4, 16, 96, 3)
    e.run()
    want = e.oracle()
    for k, got in e.outputs().items():
        off = np.linalg.norm(host(got) - want[k]) / np.linalg.norm(want[k])
        assert off <= (10 * U["bf16"] if dt == "bf16" else 2e-5), (k, off)


def test_two_captured_graphs_share_a_workspace_and_other_streams_run_beside():
    """Graphs replayed one after another on one workspace, and a run on a stream of its own with its own: the same
    bits as a run that nothing disturbs."""
    need_gpu()
    hg = lib()
    one, two = (Encoder(hg, "bf16", 5, 37 + 300 * i, 4, 32, 136, i) for i in range(2))
    if two.work.numel() > one.work.numel():
        one.work = two.work
    else:
        two.work = one.work
    want = []
    for e in (one, two):
        e.run()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in e.outputs().items()})
    side = torch.cuda.Stream()
    graphs = []
    for e in (one, two):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            e.run()
        graphs.append(g)
    other = Encoder(hg, "bf16", 5, 37, 4, 32, 136, 0)
    for e in (one, two, other):
        for v in e.outputs().values():
            v.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(3):
            for g in graphs:
                g.replay()
    own = torch.cuda.Stream()
    other.run(stream=own)
    torch.cuda.synchronize()
    for e, w in ((one, want[0]), (two, want[1]), (other, want[0])):
        for k, v in e.outputs().items():
            assert torch.equal(v, w[k]), k
    assert hg.hg_device_status() == 0
