"""Oracle of the history encoder's operators against differences and identities, and the refusals of their entry
points and binding (CPU only: fake aligned addresses stand in for device buffers, nothing is dereferenced)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import history as OH

A = 1 << 20  # a 256-byte-aligned stand-in address


@pytest.fixture(scope="module")
def hg():
    from paper_2608_02168_gb300 import build
    build.build()
    from paper_2608_02168_gb300 import hg as binding
    return binding


def central(f, x, dy, h=1e-5):
    """d <f(x), dy> / dx by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = (f() * dy).sum()
        x[i] = keep - h
        g[i] = (up - (f() * dy).sum()) / (2 * h)
        x[i] = keep
    return g


def close(a, b, tol=1e-7):
    # central differences of step 1e-5: truncation h^2 and rounding 2^-53 / h, both below 1e-9 of these values
    assert np.abs(a - b).max() <= tol * max(1.0, np.abs(b).max()), np.abs(a - b).max()


@pytest.mark.parametrize("rot,interleaved", [(16, False), (16, True), (32, False), (0, False)])
def test_rotation_gradients(rot, interleaved):
    rng = np.random.default_rng(rot)
    x, g, dy = rng.standard_normal((3, 2, 32)), rng.standard_normal(32), rng.standard_normal((3, 2, 32))
    pos = np.array([0, 5, -7])
    f = lambda: OH.qkrot_forward(x, g, pos, rot, 100.0, 1e-3, interleaved)  # noqa: E731
    dx, dg = OH.qkrot_backward(x, g, pos, rot, 100.0, 1e-3, interleaved, dy)
    close(dx, central(f, x, dy))
    close(dg, central(f, g, dy))


def test_rotation_depends_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 32))
    one = np.ones(32)
    dots = []
    for a, b in ((3, 1), (1003, 1001)):
        y = [OH.qkrot_forward(x, one, [p], 32, 1e4, 1e-6, False)[0, 0] for x, p in ((q, a), (k, b))]
        dots.append(y[0] @ y[1])
    close(np.array(dots[0]), np.array(dots[1]), 1e-10)


@pytest.mark.parametrize("lens", [None, [0, 1, 4], [4, 3, 2]])
def test_decay_gradients(lens):
    rng = np.random.default_rng(3)
    n, T, h, d = 3, 4, 2, 3
    q, k, v, do = rng.standard_normal((4, n, T, h, d))
    S, dS = rng.standard_normal((2, n, h, d, d))
    ld = np.array([-0.3, -2.0])
    lens = None if lens is None else np.array(lens)

    def both():
        o, last = OH.decay_forward(q, k, v, ld, 0.7, lens, S)
        return np.concatenate([o.ravel(), last.ravel()])

    dy = np.concatenate([do.ravel(), dS.ravel()])
    got = OH.decay_backward(q, k, v, ld, 0.7, do, lens, S, dS)
    for x, g in zip((q, k, v, S), got):
        close(g, central(both, x, dy))


def test_decay_is_the_masked_product():
    rng = np.random.default_rng(4)
    T, d = 9, 5
    q, k, v = rng.standard_normal((3, T, d))
    ld = -0.2
    gap = np.arange(T)[:, None] - np.arange(T)
    want = 0.5 * (np.where(gap >= 0, np.exp(ld * np.maximum(gap, 0)), 0.0) * (q @ k.T)) @ v
    o, S = OH.decay_forward(q[None, :, None], k[None, :, None], v[None, :, None], np.array([ld]), 0.5)
    close(o[0, :, 0], want, 1e-12)
    a, S1 = OH.decay_forward(*(x[None, :4, None] for x in (q, k, v)), np.array([ld]), 0.5)
    b, S2 = OH.decay_forward(*(x[None, 4:, None] for x in (q, k, v)), np.array([ld]), 0.5, S_in=S1)
    close(np.concatenate([a, b], 1), o, 1e-12)
    close(S2, S, 1e-12)


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "relu", "none"])
@pytest.mark.parametrize("residual", [False, True])
def test_ffn_gradients(kind, residual):
    rng = np.random.default_rng(5)
    X, dY = rng.standard_normal((2, 4, 6))
    Wg, Wu = rng.standard_normal((2, 6, 8))
    Wd = rng.standard_normal((8, 6))
    f = lambda: OH.ffn_forward(X, Wg, Wu, Wd, kind, residual)  # noqa: E731
    for x, g in zip((X, Wg, Wu, Wd), OH.ffn_backward(X, Wg, Wu, Wd, kind, residual, dY)):
        close(g, central(f, x, dY))


def test_gelu_is_torch_gelu():
    x = np.linspace(-6, 6, 101)
    want = torch.nn.functional.gelu(torch.from_numpy(x), approximate="tanh").numpy()
    close(OH.act(x, "gelu_tanh")[0], want, 1e-12)


# ---------------------------------------------------------------------------------------------- refusals
def rows(hg, p=A, stride=128):
    return ctypes.byref(hg.hg_rows(p, stride))


def seq(hg, p=A, sn=4096, st=128):
    return ctypes.byref(hg.hg_seq(p, sn, st))


def test_qkrot_refusals(hg):
    so = hg.lib()

    def params(hq=4, hk=4, dh=32, rot=32, inter=0, dt=1, eps=1e-6, base=1e4):
        return ctypes.byref(hg.hg_qkrot_params(hq, hk, dh, rot, inter, dt, eps, base, None, None))

    size = ctypes.c_size_t()

    def query(n=10, **k):
        return so.hg_qkrot_workspace_size(params(**k), n, ctypes.byref(size))

    assert query() == 0 and size.value > 0 and query(0) == 0
    assert query(dh=48) == 2 and query(dt=2) == 2 and query(dt=-1) == 2
    assert query(hq=0) == query(hq=65) == query(hk=-1) == query(hk=65) == 1
    assert query(rot=8) == query(rot=48) == query(rot=-16) == 1
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert query(eps=bad) == 1
    for bad in (0.5, float("nan"), float("inf")):
        assert query(base=bad) == 1
    assert query(-1) == 1 and so.hg_qkrot_workspace_size(None, 1, ctypes.byref(size)) == 1
    assert so.hg_qkrot_workspace_size(params(), 1, None) == 1

    def fwd(q=None, k=None, qo=None, ko=None, n=10, **kw):
        z = [rows(hg) if x is None else x for x in (q, k, qo, ko)]
        return so.hg_qkrot_fwd(params(**kw), z[0], z[1], None, n, z[2], z[3], None)

    null = ctypes.POINTER(hg.hg_rows)()
    assert fwd(q=null) == fwd(k=null) == fwd(qo=null) == fwd(ko=null) == 1
    assert fwd(q=rows(hg, A + 2)) == fwd(ko=rows(hg, A + 8)) == 1           # alignment
    assert fwd(q=rows(hg, stride=132)) == fwd(q=rows(hg, stride=-128)) == 1  # stride
    assert fwd(qo=rows(hg, stride=64)) == fwd(ko=rows(hg, stride=0)) == 1    # written rows overlap
    assert fwd(q=null, n=0) == 0

    def bwd(n=10, scratch=A, dq=None, **kw):
        r = rows(hg)
        return so.hg_qkrot_bwd(params(**kw), r, r, None, n, r, r, r if dq is None else dq, r, A, A, scratch, None)

    assert bwd(scratch=None) == bwd(scratch=A + 16) == bwd(dq=rows(hg, stride=32)) == bwd(n=-1) == 1


def test_decay_refusals(hg):
    so = hg.lib()

    def params(h=4, dh=32, dt=1, ld=A):
        return ctypes.byref(hg.hg_decay_params(h, dh, dt, 1.0, ld))

    f, b = ctypes.c_size_t(), ctypes.c_size_t()

    def query(n=3, T=5, **k):
        return so.hg_decay_workspace_size(params(**k), n, T, ctypes.byref(f), ctypes.byref(b))

    assert query() == 0 and f.value == b.value == 0
    assert query(1, 1 << 16) == 0 and f.value >= 4 * 4 * 32 * 32 * 2 and b.value >= f.value  # segments' states
    assert query(dh=24) == 2 and query(dt=7) == 2
    assert query(h=0) == query(h=65) == query(n=-1) == query(T=-1) == query(T=1 << 30) == query(n=1 << 26) == 1
    assert so.hg_decay_workspace_size(params(), 1, 1, None, ctypes.byref(b)) == 1

    def fwd(n=3, T=5, o=None, q=None, scratch=None, **kw):
        s = seq(hg)
        return so.hg_decay_fwd(params(**kw), s if q is None else q, s, s, None, n, T, None, s if o is None else o, None,
                               scratch, None)

    null = ctypes.POINTER(hg.hg_seq)()
    assert fwd(ld=None) == fwd(q=null) == fwd(o=null) == 1
    assert fwd(q=seq(hg, A + 4)) == fwd(q=seq(hg, st=-128)) == fwd(q=seq(hg, sn=4100)) == 1
    assert fwd(o=seq(hg, st=64)) == fwd(o=seq(hg, sn=512)) == fwd(o=seq(hg, sn=0)) == 1  # written rows overlap
    assert fwd(o=seq(hg, sn=128, st=256)) == 1
    assert fwd(n=1, T=1 << 16) == 1                                                      # segments need scratch
    assert fwd(n=1, T=1 << 16, scratch=A + 64) == 1
    assert fwd(n=0, q=null) == 0

    def bwd(dk=None, n=3, T=5):
        s = seq(hg)
        return so.hg_decay_bwd(params(), s, s, s, None, n, T, None, s, None, s, s if dk is None else dk, s, None, None,
                               None)

    assert bwd(dk=null) == bwd(dk=seq(hg, st=0)) == bwd(T=-1) == 1

    def step(q=None, S=A, So=A, n=3, o=None, **kw):
        r = rows(hg)
        return so.hg_decay_step(params(**kw), r if q is None else q, r, r, None, n, S, r if o is None else o, So, None)

    nullr = ctypes.POINTER(hg.hg_rows)()
    assert step(q=nullr) == step(S=None) == step(So=None) == step(So=A + 4) == step(o=rows(hg, stride=32)) == 1
    assert step(ld=None) == step(n=-1) == 1 and step(dh=20) == 2 and step(n=0, q=nullr) == 0


def test_ffn_refusals(hg):
    so = hg.lib()

    def params(d=64, f=96, dt=1, act=3, wg=A, wu=A, wd=A):
        return ctypes.byref(hg.hg_ffn_params(d, f, dt, act, 1, wg, wu, wd))

    f, b = ctypes.c_size_t(), ctypes.c_size_t()

    def query(n=10, **k):
        return so.hg_ffn_workspace_size(params(**k), n, ctypes.byref(f), ctypes.byref(b))

    assert query() == 0 and query(0) == 0
    assert query(d=96) == query(dt=3) == 2
    assert query(f=0) == query(f=12) == query(f=16392) == query(act=4) == query(act=-1) == query(-1) == 1
    assert query(1 << 31) == 1

    def fwd(X=A, Y=A, n=10, scratch=A, **kw):
        return so.hg_ffn_fwd(params(**kw), X, n, Y, scratch, None)

    assert fwd(X=None) == fwd(Y=None) == fwd(X=A + 8) == fwd(wg=None) == fwd(wd=A + 2) == 1
    assert fwd(scratch=A + 16) == 1 and fwd(X=None, n=0) == 0

    def bwd(X=A, dY=A, dX=A, n=10, g=(A, A, A), scratch=A):
        gr = None if g is None else ctypes.byref(hg.hg_ffn_grads(*g))
        return so.hg_ffn_bwd(params(), X, n, dY, dX, gr, scratch, None)

    assert bwd(g=(A, None, A)) == bwd(g=(A, A, A + 4)) == bwd(dY=None) == bwd(dX=A + 2) == bwd(scratch=None) == 1
    assert bwd(n=-1) == 1 and bwd(dX=None, g=None) == 0


def test_binding_refuses_shapes_types_and_host_tensors(hg):
    t = torch.empty(3, 2, 32)
    with pytest.raises(ValueError, match="device memory"):
        hg._heads_of(t, "q", torch.float32, (3, 2, 32))
    with pytest.raises(ValueError, match="shape"):
        hg._heads_of(t, "q", torch.float32, (3, 2, 16))
    with pytest.raises(ValueError, match="shape"):
        hg._heads_of(t, "q", torch.bfloat16, (3, 2, 32))
    with pytest.raises(ValueError, match="shape"):
        hg._want(torch.empty(3, dtype=torch.int64), "lens", torch.int32, (3,))
    with pytest.raises(ValueError, match="storage types"):
        hg._storage(torch.float16)
    with pytest.raises(ValueError, match="bytes are needed"):
        hg._work_ptr(None, 16, "scratch")
    assert hg._work_ptr(None, 0, "scratch") is None


def test_arrays_that_share_memory_are_refused(hg):
    """Outputs that start at another array's rows, each call's arrays far apart but for the one named."""
    so = hg.lib()
    P = [A + (i << 24) for i in range(8)]

    def refused(status):
        return status == 1 and b"overlap" in so.hg_last_error()

    qp = ctypes.byref(hg.hg_qkrot_params(4, 4, 32, 32, 0, 1, 1e-6, 1e4, None, None))

    def rot(q, k, qo, ko, so_stride=128):
        return so.hg_qkrot_fwd(qp, rows(hg, q), rows(hg, k), None, 10, rows(hg, qo, so_stride), rows(hg, ko), None)

    assert refused(rot(P[0], P[1], P[1], P[3])) and refused(rot(P[0], P[1], P[2], P[0]))
    assert refused(rot(P[0], P[1], P[2], P[2]))
    assert rot(P[0], P[1], P[0], P[3], so_stride=256) == 1 and b"in place" in so.hg_last_error()

    def rot_bwd(q, k, dqo, dko, dq, dk):
        r = [rows(hg, x) for x in (q, k, dqo, dko, dq, dk)]
        return so.hg_qkrot_bwd(qp, r[0], r[1], None, 10, *r[2:], None, None, A, None)

    assert refused(rot_bwd(*P[:4], P[0], P[5])) and refused(rot_bwd(*P[:4], P[4], P[1]))
    assert refused(rot_bwd(*P[:4], P[3], P[5])) and refused(rot_bwd(*P[:4], P[4], P[4]))

    dp = ctypes.byref(hg.hg_decay_params(4, 32, 1, 1.0, A))
    for i in range(3):
        s = [seq(hg, x) for x in P[:3]]
        assert refused(so.hg_decay_fwd(dp, *s, None, 3, 5, None, seq(hg, P[i]), None, None, None))
        r = [rows(hg, x) for x in P[:3]]
        assert refused(so.hg_decay_step(dp, *r, None, 3, A, rows(hg, P[i]), A, None))
    for i, j in ((4, 0), (5, 1), (6, 2), (4, 3), (5, 4), (6, 5)):
        p = P[:7]
        p[i] = P[j]
        s = [seq(hg, x) for x in p]
        assert refused(so.hg_decay_bwd(dp, *s[:3], None, 3, 5, None, s[3], None, *s[4:], None, None, None))

    fp = ctypes.byref(hg.hg_ffn_params(64, 96, 1, 3, 1, A, A, A))
    last = 9 * 128  # bytes to the last of ten rows
    for y in (P[1], P[1] + last, P[1] - last):
        assert refused(so.hg_ffn_fwd(fp, P[1], 10, y, A, None))
        assert refused(so.hg_ffn_bwd(fp, P[1], 10, P[2], y, None, A, None))
        assert refused(so.hg_ffn_bwd(fp, P[2], 10, P[1], y, None, A, None))


def test_decay_sizes_that_pass_64_bits_are_refused(hg):
    so = hg.lib()
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    p = ctypes.byref(hg.hg_decay_params(64, 32, 1, 1.0, A))
    assert so.hg_decay_workspace_size(p, 1 << 58, 5, ctypes.byref(f), ctypes.byref(b)) == 1
    # rows of the two sequences meet: the span of one, (T - 1) stride_t, is 2^66 values
    far = seq(hg, A + (1 << 30), sn=1 << 39, st=1 << 38)
    s = seq(hg)
    T = (1 << 28) + 1
    scratch = A
    assert so.hg_decay_fwd(p, s, s, s, None, 2, T, None, far, None, scratch, None) == 1
    assert b"overlap" in so.hg_last_error()


def test_decay_of_no_sequences_needs_no_scratch(hg):
    so = hg.lib()
    f, b = ctypes.c_size_t(1), ctypes.c_size_t(1)
    p = ctypes.byref(hg.hg_decay_params(4, 32, 1, 1.0, A))
    assert so.hg_decay_workspace_size(p, 0, 500, ctypes.byref(f), ctypes.byref(b)) == 0
    assert f.value == b.value == 0
    null = ctypes.POINTER(hg.hg_seq)()
    assert so.hg_decay_fwd(p, null, null, null, None, 0, 500, None, null, None, None, None) == 0


class OnDevice(torch.Tensor):
    """A host tensor that stands in for a device one: the binding reads its address, nothing is dereferenced."""
    is_cuda = True


def stand_in(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def some_params(hg):
    """Each class of parameters with its tensors by the names of its C struct."""
    f32 = torch.float32
    t = {"gamma_q": stand_in(32), "gamma_k": stand_in(32)}
    yield hg.QkRotParams(t["gamma_q"], t["gamma_k"], 4, 2), t
    t = {"log_decay": stand_in(4, dtype=f32)}
    yield hg.DecayParams(t["log_decay"], 32, torch.bfloat16), t
    t = {"W_gate": stand_in(64, 96), "W_up": stand_in(64, 96), "W_down": stand_in(96, 64)}
    yield hg.FfnParams(t["W_gate"], t["W_up"], t["W_down"]), t


def test_parameters_follow_their_tensors(hg):
    """A tensor that is given another storage is read at its new place by the next call, not where it was; another
    shape is refused."""
    for p, tensors in some_params(hg):
        for name, x in tensors.items():
            before, was = p.c(), x.data_ptr()
            assert getattr(before, name) == was
            x.data = torch.ones_like(x)
            assert x.data_ptr() != was
            assert all(getattr(p.c(), y) == tensors[y].data_ptr() for y in tensors), name
            good = x.data
            x.data = torch.zeros(*x.shape, 2, dtype=x.dtype)
            with pytest.raises(ValueError, match="shape"):
                p.c()
            x.data = torch.zeros(0, dtype=x.dtype)
            with pytest.raises(ValueError, match="shape"):
                p.c()
            x.data = good
            assert getattr(p.c(), name) == good.data_ptr()


def test_a_parameter_without_storage_is_refused(hg):
    """Its address is null, which would stand for gains of one."""
    for p, tensors in some_params(hg):
        for x in tensors.values():
            size = x.untyped_storage().nbytes()
            x.untyped_storage().resize_(0)
            with pytest.raises(ValueError, match="no storage"):
                p.c()
            x.untyped_storage().resize_(size)
            p.c()


def test_parameters_that_would_be_copies_are_refused(hg):
    """A copy of a tensor in another layout would keep the values of the moment; in-place updates reach what is taken."""
    w, g = stand_in(96, 64).t(), stand_in(64)[::2]
    assert not w.is_contiguous() and not g.is_contiguous()
    ok = stand_in(64, 96)
    for args in ((w, ok, stand_in(96, 64)), (ok, w, stand_in(96, 64)), (ok, ok.clone(), ok.t())):
        with pytest.raises(ValueError, match="must be contiguous"):
            hg.FfnParams(*args)
    with pytest.raises(ValueError, match="must be contiguous"):
        hg.QkRotParams(g, stand_in(32), 4, 4)
    with pytest.raises(ValueError, match="must be contiguous"):
        hg.QkRotParams(None, g, 4, 4)
    with pytest.raises(ValueError, match="must be contiguous"):
        hg.DecayParams(stand_in(8, dtype=torch.float32)[::2], 32, torch.bfloat16)
    assert hg.FfnParams(w.contiguous(), ok, stand_in(96, 64)).c().W_gate != w.data_ptr()


def test_rows_that_meet_without_starting_together_are_refused(hg):
    """Outputs a row, a sequence or a part of a row further on than another array; strides alike and not."""
    so = hg.lib()
    B = A + (1 << 28)

    def refused(status):
        return status == 1 and b"overlap" in so.hg_last_error()

    # rotation, 10 rows of 256 bytes (q) and 128 (k), 1024 bytes apart
    qp = ctypes.byref(hg.hg_qkrot_params(4, 2, 32, 32, 0, 1, 1e-6, 1e4, None, None))
    far = [B + (i << 22) for i in range(6)]

    def rot(q=far[0], k=far[1], qo=far[2], ko=far[3], stride=512, ostride=512):
        return so.hg_qkrot_fwd(qp, rows(hg, q, stride), rows(hg, k, stride), None, 10, rows(hg, qo, ostride),
                               rows(hg, ko, ostride), None)

    for shift in (1024, -1024, 9 * 1024, -9 * 1024, 128, -128, 5 * 1024 + 240, -5 * 1024 - 240):
        assert refused(rot(qo=far[0] + shift)), shift            # q_out over q, not in place
    for shift in (1024, -1024, 9 * 1024, -9 * 1024, 128, -112, 5 * 1024 + 240, -5 * 1024 - 112):
        assert refused(rot(ko=far[2] + shift)), shift            # k_out over q_out
    assert refused(rot(qo=far[1] + 3 * 1024 + 112)) and refused(rot(ko=far[0] - 112))
    assert refused(rot(qo=far[0] + 1024, ostride=256)) and refused(rot(qo=far[0] - 512, ostride=128))

    def rot_bwd(**k):
        p = {**dict(zip(("q", "k", "dqo", "dko", "dq", "dk"), far)), **k}
        r = [rows(hg, x, 512) for x in p.values()]
        return so.hg_qkrot_bwd(qp, r[0], r[1], None, 10, *r[2:], None, None, A, None)

    assert refused(rot_bwd(dq=far[2] + 1024)) and refused(rot_bwd(dq=far[0] + 2048)) and refused(rot_bwd(dk=far[3] - 1024))
    assert refused(rot_bwd(dk=far[4] + 1024)) and refused(rot_bwd(dk=far[2] + 9 * 1024))

    # scan, 3 sequences 8192 bytes apart of 5 rows of 256 bytes 1024 apart; and the other way round
    dp = ctypes.byref(hg.hg_decay_params(4, 32, 1, 1.0, A))
    for sn, st, one in ((4096, 512, 1024), (512, 4096, 8192)):
        def fwd(o, osn=sn, ost=st, q=far[0], sn=sn, st=st):
            s = [seq(hg, x, sn, st) for x in (q, far[1], far[2])]
            return so.hg_decay_fwd(dp, *s, None, 3, 5, None, seq(hg, o, osn, ost), None, None, None)

        for x in far[:3]:
            for shift in (one, -one, 8192, -8192, 1024, -1024, 112, -240, 2 * 8192 + 1024):
                assert refused(fwd(x + shift)), (sn, shift)
        assert refused(fwd(far[0] + 128, q=far[0], osn=640, ost=128)) and refused(fwd(far[1] + 2048, osn=128, ost=384))

        def bwd(i, x):
            p = [B + (j << 22) for j in range(7)]
            p[i] = x
            s = [seq(hg, y, sn, st) for y in p]
            return so.hg_decay_bwd(dp, *s[:3], None, 3, 5, None, s[3], None, *s[4:], None, None, None)

        for i in (4, 5, 6):
            for j in range(7):
                assert i == j or refused(bwd(i, B + (j << 22) + one)), (i, j)

    # the step's rows; states that are moved, not the same
    S, size = B + (1 << 26), 3 * 4 * 32 * 32 * 4

    def step(o=far[3], S_in=S, S_out=S):
        r = [rows(hg, x, 512) for x in far[:3]]
        return so.hg_decay_step(dp, *r, None, 3, S_in, rows(hg, o, 512), S_out, None)

    assert all(refused(step(o=x + y)) for x in far[:3] for y in (1024, -1024, 128))
    for y in (16, -16, size - 16, 16 - size):
        assert refused(step(S_out=S + y))
        s = [seq(hg, x) for x in far[:4]]
        assert refused(so.hg_decay_fwd(dp, *s[:3], None, 3, 5, S, s[3], S + y, None, None))
        g = [seq(hg, B + (j << 22)) for j in range(7)]
        for a, b in ((S, None), (None, S)):
            assert refused(so.hg_decay_bwd(dp, *g[:3], None, 3, 5, a, g[3], b, *g[4:], S + y, None, None))


def test_gradients_of_two_parameters_in_one_place_are_refused(hg):
    """Each is overwritten, none added to: one buffer for the gains of queries and keys would keep either."""
    so = hg.lib()
    P = [A + (i << 24) for i in range(8)]
    qp = ctypes.byref(hg.hg_qkrot_params(4, 4, 32, 32, 0, 1, 1e-6, 1e4, None, None))
    r = [rows(hg, x) for x in P[:6]]
    for n in (10, 0):
        for shift in (0, 4, -4, 124):
            assert so.hg_qkrot_bwd(qp, r[0], r[1], None, n, *r[2:6], P[6], P[6] + shift, A, None) == 1
            assert b"overlap" in so.hg_last_error()
    fp = ctypes.byref(hg.hg_ffn_params(64, 96, 1, 3, 1, A, A, A))
    for i, j in ((0, 1), (0, 2), (1, 2)):
        for shift in (0, 16, 64 * 96 * 4 - 16):
            g = P[:3]
            g[j] = g[i] + shift
            for n in (10, 0):
                assert so.hg_ffn_bwd(fp, P[3], n, P[4], P[5], ctypes.byref(hg.hg_ffn_grads(*g)), A, None) == 1
                assert b"overlap" in so.hg_last_error()


def test_ffn_scratch_is_asked_for_where_it_is_used(hg):
    so = hg.lib()
    g = ctypes.byref(hg.hg_ffn_grads(A, A + (1 << 20), A + (2 << 20)))
    for dt, grads in ((0, None), (0, g), (1, g)):
        p = ctypes.byref(hg.hg_ffn_params(64, 96, dt, 3, 1, A, A, A))
        assert so.hg_ffn_bwd(p, A, 10, A + (1 << 24), A + (2 << 24), grads, None, None) == 1
        assert b"scratch" in so.hg_last_error()


def test_a_parameter_turned_in_its_place_is_refused(hg):
    """The transpose of a weight has its address and size; read as it lies it would be another matrix."""
    w = stand_in(64, 64)
    p = hg.FfnParams(w, stand_in(64, 64), stand_in(64, 64))
    w.data = w.data.t()
    with pytest.raises(ValueError, match="must be contiguous"):
        p.c()
