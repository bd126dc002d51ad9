"""Gated linear recurrence (hg_recur_*) through the C ABI against the fp64 oracle.

Tolerances, element by element, with u = half a step of the storage type (2^-24 fp32, 2^-8 bf16) and s = 2^-24:
  rows and states      u |want| + (2 T + 100) s M,   M = the largest sum of absolute terms of the channel's state:
     a step rounds a difference and a sum (at most T of them, none growing: 1 - z <= 1); its logit a makes the smaller of
     z and 1 - z right to (2.4 |a| + 10) s of itself (exponential, reciprocal, the sum with the bias), and what follows is
     off by that times z |x - h| <= 2 z M with z's weights summing to at most one: below 100 s M, as |a| <= 12 where T
     gates matter at all;
  bf16 rows: 1 - z is right to 4 s of one, not of itself (z to that of itself): what it keeps, the state or R, is off by
     that of its size; summed over steps as above where z is small, and where it is not 1 - z < 1/2 keeps less than 8 s
     in all.  M is the most so far; R's sums are held at their most so far as well.
  dx                   u |want| + (2 T + 140) s A: R, a sum of at most T terms times gates, and one product;
  dg, dbias            u |want| + (4 T + 400) s A, where A takes |x| + M for the difference; dbias adds n T s A.
bf16 states and dbias are fp32: their u is 2^-24.
"""
import numpy as np
import pytest
import torch

from oracle import recur as OR
from tests.gpu_util import dev, lib, need_gpu, tdtype
from tests.test_gpu_history import F32, U, draw, f64, host, nans, near, past

pytestmark = pytest.mark.gpu


def wide(x, td, dim=-1):
    """x [n, T, d] on the device as a slice of wider rows, NaN around it."""
    shape = list(x.shape)
    d = shape[-1]
    shape[-1] = 2 * d + 8
    w = nans(shape, td)
    view = w[..., 8:8 + d]
    if x is not None:
        view.copy_(dev(x, td))
    return view


def problem(dt, n, T, d, seed, ragged, state, bias=True):
    rng = np.random.default_rng(seed)
    x, g, dy = (draw(rng, dt, n, T, d) for _ in range(3))
    b = draw(rng, dt, d, scale=2.0) if bias else None
    lens = None
    if ragged:
        lens = rng.integers(0, T + 1, n).astype(np.int32)
        lens[0], lens[-1] = 0, T
    h, dh = rng.standard_normal((2, n, d)).astype(np.float32) if state else (None, None)
    return x, g, dy, b, lens, h, dh


def params(hg, b, d, td):
    return hg.RecurParams(dev(b, td)) if b is not None else hg.RecurParams(d=d, dtype=td)


def run(hg, p, td, X, G, L, H, DY, DH, n, T, d, out=None):
    sb, wb = hg.hg_recur_workspace_size(p, n, T)
    saved = torch.full((sb,), 0xFF, dtype=torch.uint8, device="cuda")
    scratch = torch.full((wb,), 0xFF, dtype=torch.uint8, device="cuda")
    o = out or {k: nans((n, T, d), td) for k in ("y", "dx", "dg")}
    o.update({k: nans((n, d), torch.float32) for k in ("h", "dh")}, db=nans((d,), torch.float32))
    hg.hg_recur_fwd(p, X, G, L, H, o["y"], o["h"], saved)
    hg.hg_recur_bwd(p, X, G, L, H, saved, DY, DH, o["dx"], o["dg"], o["dh"], o["db"], scratch)
    return o


def check(o, dt, x, g, dy, b, lens, h, dh):
    n, T, d = x.shape
    x, g, dy, b, h, dh = (f64(v) for v in (x, g, dy, b, h, dh))
    y, last, _, most = OR.forward(x, g, b, lens, h)
    e = (2 * T + 100) * F32
    near(o["y"], y, np.broadcast_to(most[:, None], y.shape), (U[dt], e), "y")
    near(o["h"], last, most, (F32, e), "h_out")
    want, mag = OR.backward(x, g, dy, b, lens, h, dh, held=dt == "bf16")
    near(o["dx"], want["dx"], mag["dx"], (U[dt], e + 40 * F32), "dx")
    near(o["dg"], want["dg"], mag["dg"], (U[dt], 2 * e + 200 * F32), "dg")
    near(o["dh"], want["dh_in"], mag["dh_in"], (F32, e), "dh_in")
    near(o["db"], want["dbias"], mag["dbias"], (F32, 2 * e + 200 * F32 + n * T * F32), "dbias")


# a chain a thread: short histories, many histories; split over time: one to eight CTAs a cluster, tiles that end inside,
# a row of less than a piece's 32 channels, one whose last piece is not full
CASES = [(1, 1, 8, False, False), (3, 1, 64, True, True), (5, 2, 24, True, True), (300, 12, 128, True, True),
         (7, 15, 64, True, False), (4, 16, 40, False, True), (6, 17, 72, True, True), (2, 33, 520, True, True),
         (9, 64, 16, True, True), (1400, 66, 64, True, True), (3, 1030, 16384, True, True),
         (1, 65, 8, False, True), (200, 80, 64, True, True), (3, 256, 40, True, True), (4, 257, 64, True, False),
         (1, 300, 96, False, True), (2, 513, 24, True, True), (2, 1024, 64, False, False), (3, 1100, 40, True, True),
         (1, 2049, 64, False, True), (2, 4500, 8, True, True),
         (3000, 16, 24, True, True), (5000, 1, 40, False, True), (2100, 5, 264, True, False)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,d,ragged,state", CASES)
def test_forward_and_backward(dt, n, T, d, ragged, state):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, g, dy, b, lens, h, dh = problem(dt, n, T, d, n + T + d, ragged, state, bias=d % 5 != 0)
    X, G, DY = (wide(past(v, lens), td) for v in (x, g, dy))
    L, H, DH = (None if v is None else dev(v) for v in (lens, h, dh))
    out = {k: wide(np.full((n, T, d), np.nan, np.float32), td) for k in ("y", "dx", "dg")}
    o = run(hg, params(hg, b, d, td), td, X, G, L, H, DY, DH, n, T, d, out)
    check(o, dt, x, g, dy, b, lens, h, dh)
    for k in ("y", "dx", "dg"):  # what lies between the rows is left as it was
        w = o[k]._base.view(n, T, 2 * d + 8)
        assert torch.isnan(w[..., :8]).all() and torch.isnan(w[..., 8 + d:]).all(), k
        if lens is not None:
            dead = torch.arange(T, device="cuda") >= L[:, None]
            assert (o[k][dead] == 0).all(), k


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,d", [(40, 20, 64), (3, 700, 48), (700, 14, 48), (40, 7, 64)])
def test_positions_within_sequences_or_the_other_way(dt, n, T, d):
    """Rows stored position by position, [T, n, d], and inputs that one sequence's row serves (stride zero)."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, g, dy, b, lens, h, dh = problem(dt, n, T, d, 5, True, True)
    g = np.repeat(g[:1], n, 0)
    turned = lambda v: dev(np.ascontiguousarray(v.transpose(1, 0, 2)), td).transpose(0, 1)  # noqa: E731
    out = {k: nans((T, n, d), td).transpose(0, 1) for k in ("y", "dx", "dg")}
    one = dev(g[:1].copy(), td).expand(n, T, d)
    o = run(hg, params(hg, b, d, td), td, turned(x), one, dev(lens), dev(h), turned(dy), dev(dh), n, T, d, out)
    check(o, dt, x, g, dy, b, lens, h, dh)


@pytest.mark.parametrize("n,T", [(30, 40), (2, 600), (2000, 12)])
def test_optional_arguments_change_nothing_else(n, T):
    need_gpu()
    hg = lib()
    td, d = torch.bfloat16, 64
    x, g, dy, b, lens, h, dh = problem("bf16", n, T, d, 6, True, True)
    p = params(hg, b, d, td)
    X, G, DY, L, H, DH = dev(x, td), dev(g, td), dev(dy, td), dev(lens), dev(h), dev(dh)
    ref = run(hg, p, td, X, G, L, H, DY, DH, n, T, d)
    sb, wb = hg.hg_recur_workspace_size(p, n, T)
    saved = torch.empty(sb, dtype=torch.uint8, device="cuda")
    y, st = nans((n, T, d), td), H.clone()
    hg.hg_recur_fwd(p, X, G, L, st, y, st, None)  # state in place, nothing kept
    assert torch.equal(y, ref["y"]) and torch.equal(st, ref["h"])
    y = nans((n, T, d), td)
    hg.hg_recur_fwd(p, X, G, L, H, y, None, saved)
    assert torch.equal(y, ref["y"])
    dx, dg, r = nans((n, T, d), td), nans((n, T, d), td), DH.clone()
    hg.hg_recur_bwd(p, X, G, L, H, saved, DY, r, dx, dg, r, None, None)  # no bias gradient: no scratch
    assert torch.equal(dx, ref["dx"]) and torch.equal(dg, ref["dg"]) and torch.equal(r, ref["dh"])
    dx, dg = nans((n, T, d), td), nans((n, T, d), td)
    hg.hg_recur_bwd(p, X, G, L, H, saved, DY, DH, dx, dg, None, None, None)
    assert torch.equal(dx, ref["dx"]) and torch.equal(dg, ref["dg"])
    # zero states and zeros' bias are none at all; lengths past the ends are the nearer end
    zero, none = torch.zeros_like(H), params(hg, None, d, td)
    far = torch.where(L == T, 1 << 30, torch.where(L == 0, -5, L)).to(torch.int32)
    a = run(hg, none, td, X, G, L, None, DY, None, n, T, d)
    c = run(hg, hg.RecurParams(torch.zeros(d, dtype=td, device="cuda")), td, X, G, far, zero, DY, zero, n, T, d)
    for k in a:
        assert torch.equal(a[k], c[k]), k


def test_empty_calls():
    need_gpu()
    hg = lib()
    td, d = torch.bfloat16, 64
    p = params(hg, None, d, td)
    h, dh = torch.randn(5, d, device="cuda"), torch.randn(5, d, device="cuda")
    e, ho, ri, db = torch.empty(5, 0, d, dtype=td, device="cuda"), nans((5, d), torch.float32), nans((5, d), torch.float32), nans((d,), torch.float32)
    work = torch.empty(hg.hg_recur_workspace_size(p, 5, 0)[1], dtype=torch.uint8, device="cuda")
    hg.hg_recur_fwd(p, e, e, None, h, e, ho, None)  # no positions: the state passes through
    hg.hg_recur_bwd(p, e, e, None, h, None, e, dh, e, e, ri, db, work)
    assert torch.equal(ho, h) and torch.equal(ri, dh) and (db == 0).all()
    e, db = torch.empty(0, 9, d, dtype=td, device="cuda"), nans((d,), torch.float32)
    s = torch.empty(0, d, device="cuda")
    hg.hg_recur_fwd(p, e, e, None, s, e, s, None)
    hg.hg_recur_bwd(p, e, e, None, s, None, e, s, e, e, s, db, None)
    assert (db == 0).all()
    r = torch.empty(0, d, dtype=td, device="cuda")
    hg.hg_recur_step(p, r, r, None, s, r, s)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 8), (300, 128), (37, 24), (5, 16384), (1000, 2056)])
def test_step(dt, n, d):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, g, _, b, _, h, _ = problem(dt, n, 1, d, n + d, False, True)
    live = (np.random.default_rng(1).random(n) < 0.7).astype(np.int32) * 3 - (np.arange(n, dtype=np.int32) % 2)
    alive = live > 0
    p = params(hg, b, d, td)
    X, G, Y = (wide(v, td)[:, 0] for v in (x, g, np.full_like(x, np.nan)))
    X[dev(~alive)] = float("nan")
    H, out = dev(h), nans((n, d), torch.float32)
    hg.hg_recur_step(p, X, G, dev(live), H, Y, out)
    _, last, _, most = OR.forward(f64(x), f64(g), f64(b), alive.astype(int), f64(h))
    near(out, last, most, (F32, 102 * F32), "h_out")
    near(Y, last * alive[:, None], most, (U[dt], 102 * F32), "y")
    assert torch.equal(out[dev(~alive)], H[dev(~alive)]) and (Y[dev(~alive)] == 0).all()
    y2 = nans((n, d), td)
    hg.hg_recur_step(p, X, G, dev(live), H, y2)  # in place
    assert torch.equal(H, out) and torch.equal(y2, Y)
    hg.hg_recur_step(p, X[:0], G[:0], None, H[:0], y2[:0])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_history_in_one_call_in_pieces_and_snapshot_by_snapshot(dt):
    """Each is the oracle's within its own bound, so the three differ by at most twice that."""
    need_gpu()
    hg = lib()
    td, n, T, d = tdtype(dt), 3, 90, 64
    x, g, _, b, _, h, _ = problem(dt, n, T, d, 8, False, True)
    p = params(hg, b, d, td)
    X, G, H = dev(x, td), dev(g, td), dev(h)
    y, last = nans((n, T, d), td), nans((n, d), torch.float32)
    hg.hg_recur_fwd(p, X, G, None, H, y, last, None)
    _, want, _, most = OR.forward(f64(x), f64(g), f64(b), None, f64(h))
    tol = 2 * (2 * T + 101) * F32 * torch.from_numpy(most).cuda()
    s = H.clone()
    for a, z in ((0, 70), (70, 71), (71, 90)):
        hg.hg_recur_fwd(p, X[:, a:z], G[:, a:z], None, s, y[:, a:z], s, None)
    assert ((s.double() - last.double()).abs() <= tol).all()
    s = H.clone()
    for t in range(T):
        hg.hg_recur_step(p, X[:, t], G[:, t], None, s, y[:, t])
    assert ((s.double() - last.double()).abs() <= tol).all()


@pytest.mark.parametrize("n,T,d", [(70, 40, 64), (2, 900, 64)])
def test_shut_and_open_gates(n, T, d):
    """Logits of +-40 and infinite ones: z and 1 - z keep their own size.  After a state of 1e6 an open gate leaves the
    new value to a step of itself; behind shut ones a state is kept bit for bit."""
    need_gpu()
    hg = lib()
    rng = np.random.default_rng(4)
    x = draw(rng, "f32", n, T, d)
    g = rng.choice([-40.0, -12.0, 0.0, 12.0, 40.0], (n, T, d)).astype(np.float32)
    dy = draw(rng, "f32", n, T, d)
    h, dh = rng.standard_normal((2, n, d)).astype(np.float32)
    p = hg.RecurParams(d=d, dtype=torch.float32)
    o = run(hg, p, torch.float32, dev(x), dev(g), None, dev(h), dev(dy), dev(dh), n, T, d)
    check(o, "f32", x, g, dy, None, None, h, dh)
    x[:, :-1], x[:, -1] = 1e6, 1e-3
    g[:, :-1], g[:, -1] = 0.0, 40.0
    y, last = nans((n, T, d), torch.float32), nans((n, d), torch.float32)
    hg.hg_recur_fwd(p, dev(x), dev(g), None, dev(h), y, last, None)
    want = OR.forward(f64(x), f64(g), None, None, f64(h))[1]
    # the last step: 1 - z = e^-40 of a difference of 1e6, and one sum
    assert np.abs(host(last) - want).max() <= 2 * F32 * 1e-3 + 1e6 * np.exp(-40.0) * 1e-3
    for v in (-np.inf, -200.0):
        g[:] = v
        hg.hg_recur_fwd(p, dev(x), dev(g), None, dev(h), y, last, None)
        assert torch.equal(last, dev(h)) and torch.equal(y, last[:, None].expand_as(y))
    g[:] = np.inf
    hg.hg_recur_fwd(p, dev(x), dev(g), None, dev(h), y, last, None)
    assert torch.equal(y, dev(x))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,d", [(6, 40, 64), (2, 900, 64), (3, 300, 8), (6, 12, 64)])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_bad_value_reaches_nothing_before_it(dt, n, T, d, bad):
    need_gpu()
    hg = lib()
    td, t, c = tdtype(dt), 2 * T // 3, 5
    x, g, dy, b, _, h, dh = problem(dt, n, T, d, 9, False, True)
    p = params(hg, b, d, td)
    ref = run(hg, p, td, dev(x, td), dev(g, td), None, dev(h), dev(dy, td), dev(dh), n, T, d)
    x2 = x.copy()
    x2[1, t, c] = bad
    o = run(hg, p, td, dev(x2, td), dev(g, td), None, dev(h), dev(dy, td), dev(dh), n, T, d)
    hit = torch.zeros(n, T, d, dtype=torch.bool, device="cuda")
    hit[1, t:, c] = True
    assert torch.equal(o["y"][~hit], ref["y"][~hit]) and not torch.isfinite(o["y"][1, t, c]).any()
    assert torch.equal(o["dx"], ref["dx"]) and torch.equal(o["dg"][~hit], ref["dg"][~hit])
    assert torch.equal(o["dh"], ref["dh"])
    dy2 = dy.copy()
    dy2[1, t, c] = bad
    o = run(hg, p, td, dev(x, td), dev(g, td), None, dev(h), dev(dy2, td), dev(dh), n, T, d)
    hit[:] = False
    hit[1, :t + 1, c] = True
    assert torch.equal(o["y"], ref["y"])
    assert torch.equal(o["dx"][~hit], ref["dx"][~hit]) and torch.equal(o["dg"][~hit], ref["dg"][~hit])


@pytest.mark.parametrize("n,T,d", [(400, 30, 64), (2, 3000, 64), (1, 700, 40), (4000, 13, 64)])
def test_calls_repeat_their_bits_and_replay_in_a_graph(n, T, d):
    need_gpu()
    hg = lib()
    td = torch.bfloat16
    x, g, dy, b, lens, h, dh = problem("bf16", n, T, d, 10, n > 1, True)
    p = params(hg, b, d, td)
    X, G, DY, H, DH = dev(x, td), dev(g, td), dev(dy, td), dev(h), dev(dh)
    L = None if lens is None else dev(lens)
    ref = run(hg, p, td, X, G, L, H, DY, DH, n, T, d)
    for _ in range(3):
        o = run(hg, p, td, X, G, L, H, DY, DH, n, T, d)
        assert all(torch.equal(o[k], ref[k]) for k in ref)
    sb, wb = hg.hg_recur_workspace_size(p, n, T)
    saved, scratch = (torch.empty(v, dtype=torch.uint8, device="cuda") for v in (sb, wb))
    o = {k: nans(v.shape, v.dtype) for k, v in ref.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hg.hg_recur_fwd(p, X, G, L, H, o["y"], o["h"], saved)
        hg.hg_recur_bwd(p, X, G, L, H, saved, DY, DH, o["dx"], o["dg"], o["dh"], o["db"], scratch)
    for _ in range(2):
        for v in o.values():
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[k], ref[k]) for k in ref)


def test_offsets_past_32_bits():
    need_gpu()
    hg = lib()
    td, T, d = torch.bfloat16, 70, 64
    far = (1 << 32) + 64  # values between two sequences
    x, g, dy, b, _, h, dh = problem("bf16", 2, T, d, 11, False, True)
    p = params(hg, b, d, td)
    big = torch.empty(far + 5 * T * d, dtype=td, device="cuda")
    at = lambda k: torch.as_strided(big, (2, T, d), (far, d, 1), k * T * d)  # noqa: E731
    X, G, DY, y, dg = (at(k) for k in range(5))
    for view, v in ((X, x), (G, g), (DY, dy)):
        view.copy_(dev(v, td))
    o = run(hg, p, td, X, G, None, dev(h), DY, dev(dh), 2, T, d, {"y": y, "dx": nans((2, T, d), td), "dg": dg})
    ref = run(hg, p, td, dev(x, td), dev(g, td), None, dev(h), dev(dy, td), dev(dh), 2, T, d)
    assert all(torch.equal(o[k], ref[k]) for k in ref)


def test_updated_bias_is_seen():
    need_gpu()
    hg = lib()
    x, g, _, b, _, h, _ = problem("f32", 4, 9, 16, 12, False, True)
    B = dev(b)
    p = hg.RecurParams(B)
    y = nans((4, 9, 16), torch.float32)
    hg.hg_recur_fwd(p, dev(x), dev(g), None, None, y, None, None)
    B.add_(1.0)
    hg.hg_recur_fwd(p, dev(x), dev(g), None, None, y, None, None)
    want, _, _, most = OR.forward(f64(x), f64(g), f64(B.cpu().numpy()), None, None)
    near(y, want, np.broadcast_to(most[:, None], want.shape), (F32, 118 * F32), "y")


@pytest.mark.parametrize("n,T,d", [(40, 12, 64), (300, 70, 64), (3, 900, 40)])
def test_infinite_biases(n, T, d):
    """A channel that always takes its input and one that never does, with ragged histories."""
    need_gpu()
    hg = lib()
    x, g, dy, _, lens, h, dh = problem("f32", n, T, d, 13, True, True)
    b = np.zeros(d, np.float32)
    b[1], b[2] = np.inf, -np.inf
    L = dev(lens)
    o = run(hg, hg.RecurParams(dev(b)), torch.float32, dev(x), dev(g), L, dev(h), dev(dy), dev(dh), n, T, d)
    live = torch.arange(T, device="cuda") < L[:, None]
    X, H = dev(x), dev(h)
    assert torch.equal(o["y"][..., 1], X[..., 1] * live) and torch.equal(o["y"][..., 2], H[:, None, 2] * live)
    at = (L.long() - 1).clamp(min=0)[:, None]
    assert torch.equal(o["h"][:, 1], torch.where(L > 0, X[..., 1].gather(1, at)[:, 0], H[:, 1]))
    assert torch.equal(o["h"][:, 2], H[:, 2])
    assert (o["dg"][..., 1:3] == 0).all() and (o["dx"][..., 2] == 0).all() and (o["db"][1:3] == 0).all()
    keep = np.ones(d, bool)
    keep[1:3] = False
    some = {k: v[..., keep].contiguous() for k, v in o.items()}
    check(some, "f32", x[..., keep], g[..., keep], dy[..., keep], b[keep], lens, h[:, keep], dh[:, keep])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_very_long_history_and_very_many_short_ones(dt):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, g, dy, b, _, h, dh = problem(dt, 1, 100_003, 8, 14, False, True)
    o = run(hg, params(hg, b, 8, td), td, dev(x, td), dev(g, td), None, dev(h), dev(dy, td), dev(dh), 1, 100_003, 8)
    check(o, dt, x, g, dy, b, None, h, dh)
    n = 2_000_003
    gen = torch.Generator(device="cuda").manual_seed(1)
    X, G = (torch.randn(n, 2, 8, device="cuda", generator=gen).to(td) for _ in range(2))
    lens = torch.randint(0, 3, (n,), device="cuda", generator=gen).to(torch.int32)
    y, last = nans((n, 2, 8), td), nans((n, 8), torch.float32)
    hg.hg_recur_fwd(params(hg, None, 8, td), X, G, lens, None, y, last, None)
    z = torch.sigmoid(G.double())
    h0 = z[:, 0] * X[:, 0].double() * (lens > 0)[:, None]
    h1 = torch.where((lens > 1)[:, None], h0 + z[:, 1] * (X[:, 1].double() - h0), h0)
    most = X.double().abs().amax((1, 2))[:, None]
    assert ((last.double() - h1).abs() <= (2 * 2 + 100) * F32 * most).all()
    want = torch.stack([h0, h1 * (lens > 1)[:, None]], 1)
    assert ((y.double() - want).abs() <= U[dt] * want.abs() + (2 * 2 + 100) * F32 * most[:, None]).all()


@pytest.mark.parametrize("T", [20, 12])
def test_chains_with_offsets_past_32_bits(T):
    need_gpu()
    hg = lib()
    td, d = torch.bfloat16, 64
    far = (1 << 32) + 64
    x, g, dy, b, _, h, dh = problem("bf16", 2, T, d, 15, False, True)
    big = torch.empty(far + 6 * T * d, dtype=td, device="cuda")
    at = lambda k: torch.as_strided(big, (2, T, d), (far, d, 1), k * T * d)  # noqa: E731
    X, G, DY, y, dx, dg = (at(k) for k in range(6))
    for view, v in ((X, x), (G, g), (DY, dy)):
        view.copy_(dev(v, td))
    p = params(hg, b, d, td)
    o = run(hg, p, td, X, G, None, dev(h), DY, dev(dh), 2, T, d, {"y": y, "dx": dx, "dg": dg})
    ref = run(hg, p, td, dev(x, td), dev(g, td), None, dev(h), dev(dy, td), dev(dh), 2, T, d)
    assert all(torch.equal(o[k], ref[k]) for k in ref)


def test_streams_given_and_two_calls_at_once():
    """The call's stream is the one given, not the current one; calls on two streams do not meet."""
    need_gpu()
    hg = lib()
    td, n, T, d = torch.bfloat16, 3, 5000, 64
    x, g, dy, b, lens, h, dh = problem("bf16", n, T, d, 16, True, True)
    p = params(hg, b, d, td)
    X, G, L, H = dev(x, td), dev(g, td), dev(lens), dev(h)
    ref, last = nans((n, T, d), td), nans((n, d), torch.float32)
    hg.hg_recur_fwd(p, X, G, L, H, ref, last, None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[nans((n, T, d), td), nans((n, d), torch.float32)] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (y, e) in zip(streams, out):
            hg.hg_recur_fwd(p, X, G, L, H, y, e, None, stream=s)
    for s, (y, e) in zip(streams, out):
        s.synchronize()
        assert torch.equal(y, ref) and torch.equal(e, last)
    assert hg.hg_device_status() == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,T,d", [(700, 9, 520), (300, 16, 1032), (5000, 17, 24), (2000, 40, 264)])
def test_many_short_histories_of_odd_widths(dt, n, T, d):
    """More histories than threads run at once (each thread goes from one to the next), rows that several CTAs share."""
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, g, dy, b, lens, h, dh = problem(dt, n, T, d, 17, True, True)
    X, G, DY = (wide(past(v, lens), td) for v in (x, g, dy))
    out = {k: wide(np.full((n, T, d), np.nan, np.float32), td) for k in ("y", "dx", "dg")}
    o = run(hg, params(hg, b, d, td), td, X, G, dev(lens), dev(h), DY, dev(dh), n, T, d, out)
    check(o, dt, x, g, dy, b, lens, h, dh)
    for k in ("y", "dx", "dg"):
        w = o[k]._base.view(n, T, 2 * d + 8)
        assert torch.isnan(w[..., :8]).all() and torch.isnan(w[..., 8 + d:]).all(), k
