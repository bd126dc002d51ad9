"""Layer of experts (hg_moe_fwd) through the C ABI against the fp64 oracle.

Choices are equal.  Weights: within (264 + 2 |l - l_max|) steps 2^-24 of themselves (exponential, sum of up to 256, quotient;
the differences of logits are exact to a step).  Rows, with u = half a step of the storage type and s = 2^-24:
  u |want| + r A + e B,  A = the sum of |w H W_down|, B = the same with G and U by their terms' absolute values, + |x|;
r = 2^-16 in bf16 (the hidden rows as sums of two bf16 numbers), 0 in fp32; e = (3 (d + f + 40) + 4 top + 60) s: the gated block's bound
(test_gpu_history.py), the weights, and the sum over a row's experts.
"""
from fractions import Fraction

import numpy as np
import pytest
import torch

from hgsynth import bf16_round
from oracle import moe as OM
from oracle import recur as OR
from tests.gpu_util import dev, lib, need_gpu, tdtype
from tests.test_gpu_history import F32, U, draw, f64, host, nans, near

pytestmark = pytest.mark.gpu


def problem(dt, n, E, d, f, seed):
    rng = np.random.default_rng(seed)
    a = np.sqrt(2 / (d + f))
    return [draw(rng, dt, n, d), draw(rng, dt, d, E, scale=d ** -0.5), draw(rng, dt, E, d, f, scale=a),
            draw(rng, dt, E, d, f, scale=a), draw(rng, dt, E, f, d, scale=a)]


def call(hg, p, X, live=None, scratch=None):
    n = X.shape[0]
    if scratch is None:
        scratch = torch.full((hg.hg_moe_workspace_size(p, n),), 0xFF, dtype=torch.uint8, device="cuda")
    Y, e, w = nans(X.shape, X.dtype), torch.full((n, p.top_k), -7, dtype=torch.int32, device="cuda"), nans((n, p.top_k), torch.float32)
    hg.hg_moe_fwd(p, X, live, Y, e, w, scratch)
    return Y, e, w


def check(dt, got, x, ws, top, act, res, renorm, live=None):
    Y, e, w = got
    d, f = ws[1].shape[1:]
    want, idx, wt, rounded, terms = OM.forward(f64(x), *(f64(v) for v in ws), top, act, res, renorm, live)
    assert np.array_equal(e.cpu().numpy(), idx)
    l = f64(x) @ f64(ws[0])
    far = l.max(-1, keepdims=True) - np.take_along_axis(l, np.maximum(idx, 0), 1)
    near(w, wt, wt, (0, (264 + 2 * far.max(initial=0)) * F32), "weights")
    e = (3 * (d + f + 40) + 4 * top + 60) * F32
    r = 2.0**-16 if dt == "bf16" else 0
    near(Y, want, (r * rounded + e * terms) / max(r + e, 1e-30), (U[dt], r + e), "Y")


# one row, rows of one to five tiles an expert, one pass and more, chunks of f that are not full, all counts of experts,
# every width, activation and form of the weights
CASES = [(1, 1, 1, 64, 8, "silu", False, True, False), (1, 16, 2, 128, 384, "silu", True, True, False),
         (7, 3, 3, 64, 40, "relu", True, False, False), (16, 8, 2, 256, 72, "gelu_tanh", False, True, True),
         (17, 2, 1, 128, 200, "none", True, False, False), (37, 8, 2, 64, 200, "gelu_tanh", False, True, False),
         (64, 64, 2, 256, 104, "silu", True, True, False), (100, 5, 4, 128, 136, "silu", False, False, True),
         (200, 2, 2, 64, 24, "silu", True, True, False), (300, 32, 4, 256, 88, "silu", True, False, True),
         (130, 256, 8, 64, 16, "relu", False, True, False), (1024, 7, 3, 64, 56, "silu", True, True, True),
         (1000, 129, 8, 128, 32, "silu", False, False, False), (65, 1, 1, 256, 520, "silu", True, True, False),
         (4, 2, 2, 256, 136, "silu", True, True, True), (4, 9, 8, 64, 24, "gelu_tanh", False, False, False),
         (2, 2, 2, 256, 1032, "silu", True, True, False), (2, 9, 8, 128, 24, "relu", False, False, True),
         (3, 4, 3, 64, 200, "silu", True, True, False), (5, 2, 2, 256, 136, "silu", True, True, True), (64, 1, 1, 128, 40, "none", False, False, False),
         (128, 2, 2, 128, 264, "silu", False, True, False), (1024, 256, 8, 256, 8, "silu", True, False, True)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,top,d,f,act,res,renorm,masked", CASES)
def test_layer(dt, n, E, top, d, f, act, res, renorm, masked):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, *ws = problem(dt, n, E, d, f, n + E + f)
    live = (np.random.default_rng(2).random(n) < 0.7).astype(np.int32) * 2 - 1 if masked else None
    p = hg.MoeParams(*(dev(w, td) for w in ws), top, act=act, residual=res, renorm=renorm)
    X = dev(x, td)
    if masked:
        X[dev(live <= 0)] = float("nan")  # not read
    got = call(hg, p, X, None if live is None else dev(live))
    check(dt, got, x, ws, top, act, res, renorm, live)
    if masked:
        assert (got[0][dev(live <= 0)] == 0).all()
    Y = nans(X.shape, td)  # what is not wanted changes nothing
    hg.hg_moe_fwd(p, X, None if live is None else dev(live), Y, None, None,
                  torch.empty(hg.hg_moe_workspace_size(p, n), dtype=torch.uint8, device="cuda"))
    assert torch.equal(Y, got[0])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_every_row_chooses_the_same_experts(dt):
    """1000 rows of one expert: sixteen passes over its weights, and none for the others, which are not read."""
    need_gpu()
    hg = lib()
    td, n, E, d, f = tdtype(dt), 1000, 6, 64, 72
    x, wr, wg, wu, wd = problem(dt, n, E, d, f, 3)
    x[:, 0] = np.abs(x[:, 0]) + 1
    wr[:] = 0
    wr[0, 4], wr[0, 1] = 4, 2
    for w in (wg, wu, wd):
        w[[0, 2, 3, 5]] = np.nan
    p = hg.MoeParams(*(dev(w, td) for w in (wr, wg, wu, wd)), 2)
    got = call(hg, p, dev(x, td))
    for w in (wg, wu, wd):
        w[[0, 2, 3, 5]] = 0
    x = bf16_round(x) if dt == "bf16" else x  # as the device has it: the sums above are not bf16 numbers
    check(dt, got, x, (wr, wg, wu, wd), 2, "silu", False, True)
    assert (got[1] == torch.tensor([4, 1], device="cuda", dtype=torch.int32)).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_equal_logits_go_to_the_lower_index(dt):
    need_gpu()
    hg = lib()
    td, n, E, d, f = tdtype(dt), 40, 70, 64, 16
    x, wr, *ws = problem(dt, n, E, d, f, 4)
    wr[:, 35:] = wr[:, :35]
    x[3] = 0
    p = hg.MoeParams(dev(wr, td), *(dev(w, td) for w in ws), 8)
    _, e, w = call(hg, p, dev(x, td))
    e, w = e.cpu().numpy(), w.cpu().numpy()
    assert np.array_equal(e[3], np.arange(8)) and np.array_equal(w[3], np.full(8, 0.125, np.float32))
    rest = np.delete(e, 3, 0)
    assert np.array_equal(rest[:, 1::2], rest[:, ::2] + 35) and (rest[:, ::2] < 35).all()


@pytest.mark.parametrize("d", [64, 256])
def test_choices_that_rounded_logits_would_miss(d):
    """Experts that differ in the last bits of one weight, some 2^-32 of the terms' sum apart, which fp32 sums cannot
    tell: the exact ones' order."""
    need_gpu()
    hg = lib()
    rng = np.random.default_rng(5)
    n, E, f = 50, 24, 8
    x = rng.standard_normal((n, d)).astype(np.float32)
    wr = np.repeat(rng.standard_normal((d, 1)).astype(np.float32), E, 1)
    x[:, 0] = np.where(x[:, 0] < 0, -1, 1) * (1 + np.abs(x[:, 0]))
    wr[0] = 1 + rng.permutation(E).astype(np.float32) * np.float32(2.0**-23)
    ws = [rng.standard_normal(s).astype(np.float32) for s in ((E, d, f), (E, d, f), (E, f, d))]
    _, e, _ = call(hg, hg.MoeParams(dev(wr), *(dev(w) for w in ws), 5), dev(x))
    for i in range(n):
        l = [sum(Fraction(float(a)) * Fraction(float(b)) for a, b in zip(x[i], wr[:, j])) for j in range(E)]
        want = sorted(range(E), key=lambda j: (-l[j], j))
        apart = min(abs(l[a] - l[b]) for a, b in zip(want[:5], want[1:6]))
        # the bound of a sum of two numbers, twice, and as much again for the rounding of the pair
        assert apart > d * 2.0**-46 * float(np.abs(x[i]) @ np.abs(wr[:, 0]))
        assert e[i].tolist() == want[:5], i


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_row_keeps_its_own_troubles(dt, bad):
    need_gpu()
    hg = lib()
    td, n, E, d, f = tdtype(dt), 50, 4, 128, 40
    x, *ws = problem(dt, n, E, d, f, 6)
    p = hg.MoeParams(*(dev(w, td) for w in ws), 2, residual=True)
    ref = call(hg, p, dev(x, td))
    x[9, 77] = bad
    got = call(hg, p, dev(x, td))
    keep = torch.arange(n, device="cuda") != 9
    same_choice = torch.equal(got[1][9].sort()[0], ref[1][9].sort()[0])
    assert torch.equal(got[1][keep], ref[1][keep]) and torch.equal(got[2][keep], ref[2][keep])
    if same_choice:  # the same list of passes, so the same order of every sum
        assert torch.equal(got[0][keep], ref[0][keep])
    else:
        assert torch.isfinite(got[0][keep]).all()
    assert torch.isnan(got[0][9]).all() and ((got[1][9] >= 0) & (got[1][9] < E)).all()


@pytest.mark.parametrize("n,E,top,d,f", [(1, 16, 2, 128, 384), (64, 32, 2, 256, 264), (700, 9, 4, 64, 200)])
def test_calls_repeat_their_bits_and_replay_in_a_graph(n, E, top, d, f):
    """One scratch for all of them, and for another number of rows in between: the counters are each call's own."""
    need_gpu()
    hg = lib()
    td = torch.bfloat16
    x, *ws = problem("bf16", n, E, d, f, 7)
    p = hg.MoeParams(*(dev(w, td) for w in ws), top)
    X = dev(x, td)
    scratch = torch.empty(hg.hg_moe_workspace_size(p, 1024), dtype=torch.uint8, device="cuda")
    ref = call(hg, p, X, None, scratch)
    for m in (1, 5, n):
        call(hg, p, X[:m], None, scratch)
        got = call(hg, p, X, None, scratch)
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
    out = [nans(X.shape, td), torch.zeros_like(ref[1]), nans(ref[2].shape, torch.float32)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hg.hg_moe_fwd(p, X, None, *out, scratch)
    for _ in range(3):
        for v in out:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, out))


def test_no_rows_and_no_live_rows():
    need_gpu()
    hg = lib()
    td = torch.bfloat16
    x, *ws = problem("bf16", 20, 4, 64, 40, 8)
    p = hg.MoeParams(*(dev(w, td) for w in ws), 2, residual=True)
    assert hg.hg_moe_workspace_size(p, 0) == 0
    hg.hg_moe_fwd(p, torch.empty(0, 64, dtype=td, device="cuda"), None, torch.empty(0, 64, dtype=td, device="cuda"), None,
                  None, None)
    Y, e, w = call(hg, p, nans((20, 64), td), torch.zeros(20, dtype=torch.int32, device="cuda"))
    assert (Y == 0).all() and (e == -1).all() and (w == 0).all()


def test_weights_past_32_bits_of_bytes():
    need_gpu()
    hg = lib()
    td, n, E, d, f = torch.bfloat16, 3, 256, 256, 16384
    x, wr, wg, wu, wd = problem("bf16", n, 1, d, f, 9)
    big = [torch.zeros(E, *s, dtype=td, device="cuda") for s in ((d, f), (d, f), (f, d))]
    for t, w in zip(big, (wg, wu, wd)):
        t[255].copy_(dev(w[0], td))
    r = np.zeros((d, E), np.float32)
    x[:, 0] = np.abs(x[:, 0]) + 1
    r[0, 255] = 1
    Y, e, _ = call(hg, hg.MoeParams(dev(r, td), *big, 1), dev(x, td))
    assert (e == 255).all()
    one = call(hg, hg.MoeParams(dev(r[:, 255:].copy(), td), *(t[255:] for t in big), 1), dev(x, td))
    assert torch.equal(one[0], Y)
    check("bf16", one, bf16_round(x), (r[:, 255:], wg, wu, wd), 1, "silu", False, True)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_new_snapshot_through_the_recurrence_and_the_experts(dt):
    """What scoring does: the recurrence's step on the nodes with a new snapshot, then the experts on its rows, captured
    once and replayed.  The layer is checked on the rows that the step wrote."""
    need_gpu()
    hg = lib()
    td, n, d, E, f = tdtype(dt), 60, 64, 8, 72
    rng = np.random.default_rng(10)
    x, g = draw(rng, dt, n, d), draw(rng, dt, n, d)
    h = rng.standard_normal((n, d)).astype(np.float32)
    live = (rng.random(n) < 0.8).astype(np.int32)
    _, *ws = problem(dt, n, E, d, f, 11)
    rp, mp = hg.RecurParams(d=d, dtype=td), hg.MoeParams(*(dev(w, td) for w in ws), 2, residual=True)
    X, G, H, L = dev(x, td), dev(g, td), dev(h), dev(live)
    y, out, Y = nans((n, d), td), nans((n, d), torch.float32), nans((n, d), td)
    e, w = torch.zeros(n, 2, dtype=torch.int32, device="cuda"), nans((n, 2), torch.float32)
    scratch = torch.empty(hg.hg_moe_workspace_size(mp, n), dtype=torch.uint8, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        hg.hg_recur_step(rp, X, G, L, H, y, out)
        hg.hg_moe_fwd(mp, y, L, Y, e, w, scratch)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    _, last, _, most = OR.forward(f64(x)[:, None], f64(g)[:, None], None, live, f64(h))
    near(out, last, most, (F32, 102 * F32), "h_out")
    check(dt, (Y, e, w), host(y), ws, 2, "silu", True, True, live)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_the_layer_is_the_blocks_on_each_experts_rows(dt):
    """What training does with the choice: hg_ffn_fwd on each expert's rows, weighted and summed.  Both forms are within
    their bounds of the same numbers; a block's rows are rounded once more."""
    need_gpu()
    hg = lib()
    td, n, d, E, f, top = tdtype(dt), 90, 64, 5, 40, 2
    x, *ws = problem(dt, n, E, d, f, 12)
    W = [dev(w, td) for w in ws]
    p, X = hg.MoeParams(*W, top), dev(x, td)
    Y, e, w = call(hg, p, X)
    total = torch.zeros(n, d, dtype=torch.float64, device="cuda")
    for k in range(E):
        rows, j = (e == k).nonzero(as_tuple=True)
        if len(rows) == 0:
            continue
        fp = hg.FfnParams(W[1][k], W[2][k], W[3][k])
        out = nans((len(rows), d), td)
        scratch = torch.empty(max(1, hg.hg_ffn_workspace_size(fp, len(rows))[0]), dtype=torch.uint8, device="cuda")
        hg.hg_ffn_fwd(fp, X[rows].contiguous(), out, scratch)
        total.index_add_(0, rows, out.double() * w[rows, j].double()[:, None])
    _, _, _, rounded, terms = OM.forward(f64(x), *(f64(v) for v in ws), top, "silu", False, True)
    e = (3 * (d + f + 40) + 4 * top + 60) * F32
    r = U["bf16"] if dt == "bf16" else 0
    near(Y, host(total), 2 * (r * rounded + e * terms) + U[dt] * rounded, (U[dt], 1.0), "Y")


def test_streams_given_and_two_calls_at_once():
    need_gpu()
    hg = lib()
    td, n, E, d, f = torch.bfloat16, 90, 12, 128, 264
    x, *ws = problem("bf16", n, E, d, f, 13)
    p, X = hg.MoeParams(*(dev(w, td) for w in ws), 3), dev(x, td)
    ref = call(hg, p, X)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [torch.empty(hg.hg_moe_workspace_size(p, n), dtype=torch.uint8, device="cuda") for _ in streams]
    out = [[nans(X.shape, td), torch.zeros_like(ref[1]), nans(ref[2].shape, torch.float32)] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, w, o in zip(streams, work, out):
            hg.hg_moe_fwd(p, X, None, *o, w, stream=s)
    for s, o in zip(streams, out):
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o, ref))
    assert hg.hg_device_status() == 0


def test_updated_weights_are_seen():
    need_gpu()
    hg = lib()
    x, *ws = problem("f32", 9, 4, 64, 40, 14)
    W = [dev(w) for w in ws]
    p, X = hg.MoeParams(*W, 2), dev(x)
    call(hg, p, X)
    for w in W:
        w.mul_(-0.5)
    check("f32", call(hg, p, X), x, [w.cpu().numpy() for w in W], 2, "silu", False, True)
