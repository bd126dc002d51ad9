"""What is measured of the history encoder's operators: calls over the range of a node's or a user's history.

A node's history is a sequence of T snapshots (or of T events) of width d, split into heads of width d_h.  "op" says
which operator a case calls:
  qkrot  RMS norm of each query and key head with a gain, and the rotation by the snapshot's position, in one pass
  decay  causal linear attention with a decay for each head over whole histories, from and to a carried state
  step   the same for one new snapshot of every node: the carried state is read, updated and written
  ffn    gated feed-forward block: (act(X W_gate) * (X W_up)) W_down, and the residual
and "dir" whether the call is the forward or the backward pass.

Definitions (t counts snapshots from 0, gamma = exp(log_decay[head]), c = scale):
  qkrot  n = x / sqrt(mean(x^2) + eps) * gain;  pairs (i, i + rot / 2) (or (2i, 2i + 1)), i < rot / 2, are turned by
         the angle pos * base^(-2 i / rot); features from rot on stay as they are
  decay  S_t = gamma S_(t-1) + k_t v_t^T,  o_t = c q_t S_t,  S_(-1) = the state given; positions from a sequence's
         length on give zero rows and leave the state as it is
  ffn    Y = (act(X W_gate) * (X W_up)) W_down (+ X)
"""
import math

import torch

own = False

DEV = "cuda"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # scoring: queries and keys of 300 nodes' new snapshots, positions in days (latency)
        {"name": "qkrot-300", "op": "qkrot", "dir": "fwd", "n": 300, "hq": 4, "hk": 4, "dh": 32, "rot": 32,
         "pairs": "halves", "far": True, "dtype": "bf16"},
        # training: the backward pass over the histories of a large batch, d = 128
        {"name": "qkrot-bwd-1m", "op": "qkrot", "dir": "bwd", "n": 1_000_003, "hq": 4, "hk": 4, "dh": 32, "rot": 32,
         "pairs": "halves", "far": False, "dtype": "bf16"},
        # fp32, wide heads, fewer key heads, half of the features turned, event times in seconds
        {"name": "qkrot-f32", "op": "qkrot", "dir": "fwd", "n": 200_001, "hq": 4, "hk": 2, "dh": 64, "rot": 32,
         "pairs": "interleaved", "far": True, "dtype": "f32"},
        # a new snapshot of 300 nodes (latency)
        {"name": "step-300", "op": "step", "dir": "fwd", "n": 300, "heads": 4, "dh": 32, "live": 1.0,
         "dtype": "bf16"},
        # a new snapshot of 200k nodes, one in eight of them without one
        {"name": "step-200k", "op": "step", "dir": "fwd", "n": 200_000, "heads": 4, "dh": 32, "live": 0.875,
         "dtype": "bf16"},
        # snapshot histories of 150k nodes, up to 12 snapshots, ragged
        {"name": "decay-short", "op": "decay", "dir": "fwd", "n": 150_001, "T": 12, "heads": 4, "dh": 32,
         "ragged": True, "state": False, "dtype": "bf16"},
        # event histories of a few heavy users, d = 256
        {"name": "decay-long", "op": "decay", "dir": "fwd", "n": 6, "T": 32_768, "heads": 4, "dh": 64,
         "ragged": False, "state": True, "dtype": "bf16"},
        # training over event histories, d = 256, ragged
        {"name": "decay-bwd", "op": "decay", "dir": "bwd", "n": 400, "T": 515, "heads": 4, "dh": 64,
         "ragged": True, "state": True, "dtype": "bf16"},
        # the block on 300 rows (latency)
        {"name": "ffn-300", "op": "ffn", "dir": "fwd", "n": 300, "d": 128, "f": 384, "act": "silu", "res": True,
         "dtype": "bf16"},
        # the block on a large batch at the widest d
        {"name": "ffn-1m", "op": "ffn", "dir": "fwd", "n": 1_000_003, "d": 256, "f": 704, "act": "silu", "res": True,
         "dtype": "bf16"},
        # training step of the block, d = 128
        {"name": "ffn-bwd", "op": "ffn", "dir": "bwd", "n": 400_003, "d": 128, "f": 384, "act": "silu", "res": True,
         "dtype": "bf16"},
        # the same in fp32 at d = 64, GELU gate
        {"name": "ffn-bwd-f32", "op": "ffn", "dir": "bwd", "n": 20_011, "d": 64, "f": 200, "act": "gelu_tanh",
         "res": False, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qkrot", "decay", "decay", "step", "ffn", "ffn"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    way = rng.choice(["fwd", "bwd"])
    f32 = dtype == "f32"
    if op == "qkrot":
        dh = rng.choice([16, 32, 32, 64, 128])
        hq = rng.choice([1, 2, 4, 8])
        width = dh * hq
        return {"op": op, "dir": way, "n": _log(rng, 1, 60_000_000 // width), "hq": hq,
                "hk": rng.choice([hq, hq, max(1, hq // 2), 1]), "dh": dh, "rot": rng.choice([dh, dh, 16, 0]),
                "pairs": rng.choice(["halves", "interleaved"]), "far": rng.random() < 0.5, "dtype": dtype}
    if op == "step":
        dh = rng.choice([16, 32, 32, 64, 128])
        heads = rng.choice([1, 2, 4])
        return {"op": op, "dir": "fwd", "n": _log(rng, 1, 400_000_000 // (heads * dh * dh)), "heads": heads, "dh": dh,
                "live": rng.choice([1.0, 0.9, 0.5]), "dtype": dtype}
    if op == "decay":
        dh = rng.choice([16, 32, 32, 64, 64, 128])
        heads = rng.choice([1, 2, 4, 4])
        T = _log(rng, 1, 16_000)
        most = (30_000_000 if f32 else 100_000_000) // (heads * dh * T)
        return {"op": op, "dir": way, "n": _log(rng, 1, max(1, min(most, 200_000_000 // (heads * dh * dh)))), "T": T,
                "heads": heads, "dh": dh, "ragged": rng.random() < 0.5, "state": rng.random() < 0.5, "dtype": dtype}
    d = rng.choice([64, 128, 128, 256])
    f = 8 * rng.randint(d // 8, d // 2)
    most = (10 if f32 else 50 if way == "bwd" else 150) * 1_000_000_000 // (d * f)
    return {"op": op, "dir": way, "n": _log(rng, 1, most), "d": d, "f": f,
            "act": rng.choice(["silu", "silu", "gelu_tanh", "relu", "none"]), "res": rng.random() < 0.5,
            "dtype": dtype}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    td = TD[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=td):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    s = {"case": dict(case)}
    if case["op"] == "qkrot":
        # queries and keys as a projection writes them, one row for a token: [queries | keys | values]
        n, hq, hk, dh = case["n"], case["hq"], case["hk"], case["dh"]
        x = normal(n, (hq + 2 * hk) * dh)
        s["q"] = x[:, :hq * dh].unflatten(1, (hq, dh))
        s["k"] = x[:, hq * dh:(hq + hk) * dh].unflatten(1, (hk, dh))
        s["gq"], s["gk"] = ((1 + 0.1 * normal(dh, dtype=torch.float32)).to(td) for _ in range(2))
        s["pos"] = torch.randint(0, 1 << 31 if case["far"] else 512, (n,), generator=g, device=DEV)
        if case["dir"] == "bwd":
            s["dyq"], s["dyk"] = normal(n, hq, dh), normal(n, hk, dh)
        return s
    if case["op"] in ("decay", "step"):
        n, h, dh = case["n"], case["heads"], case["dh"]
        # memories from a few snapshots to a few hundred; queries and keys as the norm gives them
        s["ld"] = torch.log1p(-torch.exp2(-2.0 - 6.0 * torch.arange(h, device=DEV) / h)).float()
        s["scale"] = dh ** -0.5
        if case["op"] == "step":
            s["q"], s["k"], s["v"] = (normal(n, h, dh) for _ in range(3))
            s["state"] = normal(n, h, dh, dh, dtype=torch.float32)
            s["live"] = (torch.rand(n, generator=g, device=DEV) < case["live"]).to(torch.int32)
            return s
        T = case["T"]
        s["q"], s["k"], s["v"] = normal(n, T, 3, h, dh).unbind(2)
        s["lens"] = torch.randint(0, T + 1, (n,), generator=g, device=DEV).to(torch.int32) if case["ragged"] else None
        s["s0"] = normal(n, h, dh, dh, dtype=torch.float32) if case["state"] else None
        if case["dir"] == "bwd":
            s["do"] = normal(n, T, h, dh)
            s["ds"] = normal(n, h, dh, dh, dtype=torch.float32) if case["state"] else None
        return s
    n, d, f = case["n"], case["d"], case["f"]
    s["x"] = normal(n, d)
    a, b = math.sqrt(2 / (d + f)), math.sqrt(2 / (d + f))
    s["wg"], s["wu"], s["wd"] = normal(d, f, scale=a), normal(d, f, scale=a), normal(f, d, scale=b)
    if case["dir"] == "bwd":
        s["dy"] = normal(n, d)
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms (32 bits, one rounding at the end; angles in 64 bits)
# ---------------------------------------------------------------------------------------------------------------
def _turn(x, pos, rot, pairs, back=False):
    """Pairs of the first `rot` features of x (n x heads x d_h) turned by pos * base^(-2 i / rot)."""
    if rot == 0:
        return x
    freq = BASE ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    ang = pos.double()[:, None, None] * freq
    cos, sin = ang.cos().to(x.dtype), ang.sin().to(x.dtype)
    sin = -sin if back else sin
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if pairs == "halves" else (x[..., 0:rot:2], x[..., 1:rot:2])
    y0, y1 = a * cos - b * sin, b * cos + a * sin
    y = torch.cat([y0, y1], -1) if pairs == "halves" else torch.stack([y0, y1], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _norm_turn(x, gain, pos, rot, pairs, dtype):
    x, gain = x.to(dtype), gain.to(dtype)
    return _turn(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain, pos, rot, pairs)


def _norm_turn_bwd(x, gain, pos, rot, pairs, dy, dtype):
    x, gain = x.to(dtype), gain.to(dtype)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    g = _turn(dy.to(dtype), pos, rot, pairs, back=True)
    a = g * gain
    dx = r * a - r ** 3 * x * (a * x).mean(-1, keepdim=True)
    return dx, (g * x * r).sum((0, 1))


def _scan(q, k, v, ld, lens, init, shift):
    """Rows o_t = q_t (gamma^(t + shift) init + sum_(u <= t) gamma^(t - u) k_u v_u^T) and the state after the last
    one, times gamma for shift 0.  Chunks of 64: products within a chunk, states between chunks."""
    n, T, h, d = q.shape
    C = min(T, 64)
    nc = -(-T // C)
    t = torch.arange(T, device=DEV)
    live = torch.ones(n, T, device=DEV, dtype=torch.bool) if lens is None else t < lens[:, None]
    ends = torch.full((n,), T, device=DEV) if lens is None else lens.long()
    q, k, v = (torch.where(live[:, :, None, None], x, 0.0) for x in (q, k, v))

    left = (ends[:, None] - 1 - t).clamp(min=0)
    w = torch.exp(ld[None, None, :] * (left + (1 - shift))[:, :, None])
    last = torch.einsum("nthi,nthj->nhij", k * w[..., None], v)
    if init is not None:
        last = last + init * torch.exp(ld[None, :] * ends[:, None])[:, :, None, None]

    def chunks(x):
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, nc * C - T))
        return x.unflatten(1, (nc, C)).permute(0, 3, 1, 2, 4)

    q, k, v = chunks(q), chunks(k), chunks(v)
    i = torch.arange(C, device=DEV)
    gap = i[:, None] - i
    D = torch.where(gap >= 0, torch.exp(ld[:, None, None] * gap.clamp(min=0)), 0.0)
    o = ((q @ k.transpose(-1, -2)) * D[:, None]) @ v
    if nc > 1 or init is not None:
        local = (k * torch.exp(ld[:, None] * (C - 1 - i))[:, None, :, None]).transpose(-1, -2) @ v
        c = torch.arange(nc, device=DEV)
        gap = C * (c[:, None] - 1 - c) + (1 - shift)
        M = torch.where(c[:, None] > c, torch.exp(ld[:, None, None] * gap.clamp(min=0)), 0.0)
        enter = torch.einsum("hce,nheij->nhcij", M, local)
        if init is not None:
            enter = enter + torch.exp(ld[:, None] * (C * c))[:, :, None, None] * init[:, :, None]
        o = o + (q * torch.exp(ld[:, None] * (i + shift))[:, None, :, None]) @ enter
    o = o.permute(0, 2, 3, 1, 4).reshape(n, nc * C, h, d)[:, :T]
    return torch.where(live[:, :, None, None], o, 0.0), last


def _back(x, lens):
    """x (n x T x ...) with each sequence's own positions in reverse order."""
    T = x.shape[1]
    if lens is None:
        return x.flip(1)
    at = (lens.long()[:, None] - 1 - torch.arange(T, device=DEV)).clamp(min=0)
    return torch.gather(x, 1, at[:, :, None, None].expand_as(x))


def _decay(s):
    q, k, v = (s[x].float() for x in "qkv")
    o, last = _scan(q * s["scale"], k, v, s["ld"], s["lens"], s["s0"], 1)
    return {"o": o.to(s["q"].dtype), "state": last}


def _decay_bwd(s):
    """dq_t = c S_t do_t; with R_t = gamma R_(t+1) + c q_t do_t^T: dk_t = R_t v_t, dv_t = R_t^T k_t."""
    q, k, v, do = (s[x].float() for x in ("q", "k", "v", "do"))
    ld, lens, c, ds = s["ld"], s["lens"], s["scale"], s["ds"]
    swap = lambda x: None if x is None else x.transpose(-1, -2)  # noqa: E731
    dq, _ = _scan(do * c, v, k, ld, lens, swap(s["s0"]), 1)
    qr, kr, vr, gr = (_back(x, lens) for x in (q * c, k, v, do))
    dk, _ = _scan(vr, gr, qr, ld, lens, swap(ds), 0)
    dv, ds0 = _scan(kr, qr, gr, ld, lens, ds, 0)
    live = 1.0 if lens is None else (torch.arange(q.shape[1], device=DEV) < lens[:, None])[:, :, None, None]
    out = {"dq": dq, "dk": _back(dk, lens) * live, "dv": _back(dv, lens) * live}
    out = {x: y.to(s["q"].dtype) for x, y in out.items()}
    return {**out, "dstate": ds0}


def _step(s):
    q, k, v = (s[x].float() for x in "qkv")
    live = s["live"].bool()
    new = s["state"] * torch.exp(s["ld"])[:, None, None] + k[..., :, None] * v[..., None, :]
    o = s["scale"] * (q[..., :, None] * new).sum(-2)
    o = torch.where(live[:, None, None], o, 0.0)
    return {"o": o.to(s["q"].dtype), "state": torch.where(live[:, None, None, None], new, s["state"])}


def _act(g, kind):
    """act(g) and its derivative."""
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    if kind == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    return g, torch.ones_like(g)


def _ffn(x, wg, wu, wd, kind, res, dtype):
    x, wg, wu, wd = (y.to(dtype) for y in (x, wg, wu, wd))
    y = (_act(x @ wg, kind)[0] * (x @ wu)) @ wd
    return y + x if res else y


def _ffn_bwd(x, wg, wu, wd, dy, kind, res, dtype):
    x, wg, wu, wd, dy = (y.to(dtype) for y in (x, wg, wu, wd, dy))
    u = x @ wu
    a, da = _act(x @ wg, kind)
    dh = dy @ wd.T
    dg, du = dh * u * da, dh * a
    dx = dg @ wg.T + du @ wu.T
    return {"dx": dx + dy if res else dx, "dwg": x.T @ dg, "dwu": x.T @ du, "dwd": (a * u).T @ dy}


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if own:
        return _own(s)
    td = TD[c["dtype"]]
    if c["op"] == "qkrot":
        how = (s["pos"], c["rot"], c["pairs"])
        if c["dir"] == "fwd":
            return {x: _norm_turn(s[x], s["g" + x], *how, torch.float32).to(td) for x in "qk"}
        (dq, gq), (dk, gk) = (_norm_turn_bwd(s[x], s["g" + x], *how, s["dy" + x], torch.float32) for x in "qk")
        return {"dq": dq.to(td), "dk": dk.to(td), "dgq": gq, "dgk": gk}
    if c["op"] == "step":
        return _step(s)
    if c["op"] == "decay":
        return _decay(s) if c["dir"] == "fwd" else _decay_bwd(s)
    w = (s["x"], s["wg"], s["wu"], s["wd"])
    if c["dir"] == "fwd":
        return _ffn(*w, c["act"], c["res"], torch.float32).to(td)
    out = _ffn_bwd(*w, s["dy"], c["act"], c["res"], torch.float32)
    return {**out, "dx": out["dx"].to(td)}


def _plan(s):
    """What a program keeps for calls of one shape: parameters, workspace, output buffers."""
    from paper_2608_02168_gb300 import hg
    c, td = s["case"], TD[s["case"]["dtype"]]
    new = lambda *shape, dtype=td: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    work = lambda b: torch.empty(b, dtype=torch.uint8, device=DEV)  # noqa: E731
    if c["op"] == "qkrot":
        p = hg.QkRotParams(s["gq"], s["gk"], c["hq"], c["hk"], rot=c["rot"], base=BASE, eps=EPS,
                           interleaved=c["pairs"] == "interleaved")
        out = {"q": new(*s["q"].shape), "k": new(*s["k"].shape)}
        if c["dir"] == "fwd":
            return hg, p, out, None
        f = {x: new(c["dh"], dtype=torch.float32) for x in ("gamma_q", "gamma_k")}
        return hg, p, {**out, **f}, work(hg.hg_qkrot_workspace_size(p, c["n"]))
    if c["op"] in ("decay", "step"):
        p = hg.DecayParams(s["ld"], c["dh"], td, scale=s["scale"])
        if c["op"] == "step":
            return hg, p, {"o": new(*s["q"].shape), "state": torch.empty_like(s["state"])}, None
        st = new(c["n"], c["heads"], c["dh"], c["dh"], dtype=torch.float32)
        fwd, bwd = hg.hg_decay_workspace_size(p, c["n"], c["T"])
        row = s["q"].shape
        if c["dir"] == "fwd":
            return hg, p, {"o": new(*row), "state": st}, work(fwd)
        return hg, p, {"dq": new(*row), "dk": new(*row), "dv": new(*row), "dstate": st}, work(bwd)
    p = hg.FfnParams(s["wg"], s["wu"], s["wd"], act=c["act"], residual=c["res"])
    fwd, bwd = hg.hg_ffn_workspace_size(p, c["n"])
    if c["dir"] == "fwd":
        return hg, p, {"y": new(c["n"], c["d"])}, work(fwd)
    f = {"W_gate": (c["d"], c["f"]), "W_up": (c["d"], c["f"]), "W_down": (c["f"], c["d"])}
    return hg, p, {"dx": new(c["n"], c["d"]), **{k: new(*v, dtype=torch.float32) for k, v in f.items()}}, work(bwd)


def _own(s):
    c = s["case"]
    if "plan" not in s:
        s["plan"] = _plan(s)
    hg, p, o, w = s["plan"]
    if c["op"] == "qkrot":
        if c["dir"] == "fwd":
            hg.hg_qkrot_fwd(p, s["q"], s["k"], s["pos"], o["q"], o["k"])
            return o
        hg.hg_qkrot_bwd(p, s["q"], s["k"], s["pos"], s["dyq"], s["dyk"], o["q"], o["k"], o, w)
        return {"dq": o["q"], "dk": o["k"], "dgq": o["gamma_q"], "dgk": o["gamma_k"]}
    if c["op"] == "step":
        hg.hg_decay_step(p, s["q"], s["k"], s["v"], s["live"], s["state"], o["o"], o["state"])
        return o
    if c["op"] == "decay":
        if c["dir"] == "fwd":
            hg.hg_decay_fwd(p, s["q"], s["k"], s["v"], s["lens"], s["s0"], o["o"], o["state"], w)
            return o
        hg.hg_decay_bwd(p, s["q"], s["k"], s["v"], s["lens"], s["s0"], s["do"], s["ds"], o["dq"], o["dk"], o["dv"],
                        o["dstate"], w)
        return o
    if c["dir"] == "fwd":
        hg.hg_ffn_fwd(p, s["x"], o["y"], w)
        return o["y"]
    hg.hg_ffn_bwd(p, s["x"], s["dy"], o["dx"], o, w)
    return {"dx": o["dx"], "dwg": o["W_gate"], "dwu": o["W_up"], "dwd": o["W_down"]}


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    bwd = case["dir"] == "bwd"
    if case["op"] == "qkrot":
        rows = case["n"] * (case["hq"] + case["hk"])
        return {"bytes": rows * case["dh"] * b * (3 if bwd else 2) + 8 * case["n"],
                "flops": rows * case["dh"] * (14 if bwd else 7)}
    if case["op"] in ("step", "decay"):
        n, h, dh = case["n"], case["heads"], case["dh"]
        state = n * h * dh * dh * 4
        if case["op"] == "step":
            return {"bytes": 2 * state + 4 * n * h * dh * b, "flops": 4 * n * h * dh * dh}
        tokens = n * case["T"] * (0.5 if case["ragged"] else 1.0)
        states = state * ((2 if case["state"] else 1) + (1 if bwd and case["state"] else 0))
        # rows read up to a sequence's length, rows written up to T
        rows = tokens * (4 if bwd else 3) + n * case["T"] * (3 if bwd else 1)
        return {"bytes": rows * h * dh * b + states, "flops": tokens * h * dh * dh * (12 if bwd else 4)}
    n, d, f = case["n"], case["d"], case["f"]
    weights = 3 * d * f
    if bwd:  # the two projections again, the hidden gradient, two products into dX, three into the weights
        return {"bytes": 3 * n * d * b + weights * (b + 4), "flops": 16 * n * d * f}
    return {"bytes": 2 * n * d * b + weights * b, "flops": 6 * n * d * f}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_qkrot(s, c):
    """Complex numbers: a pair is one number, a turn is one product."""
    pos, rot, dh = s["pos"].double(), c["rot"], c["dh"]
    e = torch.arange(0, rot, 2, device=DEV, dtype=torch.float64)
    turn = torch.polar(torch.ones((), device=DEV, dtype=torch.float64).expand(len(pos), rot // 2),
                       pos[:, None] * torch.pow(torch.tensor(BASE, device=DEV, dtype=torch.float64), -e / rot))
    order = torch.arange(dh, device=DEV)  # the order in which the features of a pair are neighbours
    if c["pairs"] == "halves":
        order[:rot] = order[:rot].view(2, rot // 2).T.reshape(-1)
    undo = torch.argsort(order)

    def rotate(x, z):
        x = x[..., order]
        w = torch.view_as_complex(x[..., :rot].unflatten(-1, (rot // 2, 2)).contiguous()) * z[:, None, :]
        return torch.cat([torch.view_as_real(w).flatten(-2), x[..., rot:]], -1)[..., undo]

    def unit(x):
        ms = (x * x).sum(-1, keepdim=True) / dh + EPS
        return x / ms.sqrt(), ms

    if c["dir"] == "fwd":
        return {x: rotate(unit(s[x].double())[0] * s["g" + x].double(), turn) for x in "qk"}
    out = {}
    for x in "qk":
        u, ms = unit(s[x].double())
        g = rotate(s["dy" + x].double(), turn.conj())
        a = g * s["g" + x].double()
        out["d" + x] = (a - u * (a * u).sum(-1, keepdim=True) / dh) / ms.sqrt()
        out["dg" + x] = (g * u).flatten(0, 1).sum(0)
    return {k: out[k] for k in ("dq", "dk", "dgq", "dgk")}


def _exact_decay(s, c):
    """The recurrence, one position after another."""
    n, T, h, dh = s["q"].shape
    decay = torch.exp(s["ld"].double())[:, None, None]
    lens = torch.full((n,), T, device=DEV) if s["lens"] is None else s["lens"]
    zero = lambda x: torch.zeros(n, h, dh, dh, device=DEV, dtype=torch.float64) if x is None else x.double()  # noqa: E731
    row = lambda x, t: s[x][:, t].double()  # noqa: E731
    outer = lambda a, b: a[..., :, None] * b[..., None, :]  # noqa: E731
    state = zero(s["s0"])
    o = torch.zeros(n, T, h, dh, device=DEV, dtype=torch.float64)
    for t in range(T):
        live = (t < lens).view(n, 1, 1)
        state = torch.where(live[..., None], decay * state + outer(row("k", t), row("v", t)), state)
        if c["dir"] == "fwd":
            y = (row("q", t)[..., None, :] @ state)[..., 0, :]
        else:
            y = (state @ row("do", t)[..., None])[..., 0]
        o[:, t] = torch.where(live, s["scale"] * y, 0.0)
    if c["dir"] == "fwd":
        return {"o": o, "state": state}
    dk, dv = torch.zeros_like(o), torch.zeros_like(o)
    R = zero(s["ds"])
    for t in reversed(range(T)):
        live = (t < lens).view(n, 1, 1)
        now = R + s["scale"] * outer(row("q", t), row("do", t))
        dk[:, t] = torch.where(live, (now @ row("v", t)[..., None])[..., 0], 0.0)
        dv[:, t] = torch.where(live, (row("k", t)[..., None, :] @ now)[..., 0, :], 0.0)
        R = torch.where(live[..., None], decay * now, R)
    return {"dq": o, "dk": dk, "dv": dv, "dstate": R}


def _exact_ffn(s, c):
    """The forward in 64 bits; the gradients from its derivative as torch takes it."""
    names = ("x", "wg", "wu", "wd")
    t = {k: s[k].double().requires_grad_(c["dir"] == "bwd") for k in names}
    g = t["x"] @ t["wg"]
    if c["act"] == "silu":
        a = g / (1 + torch.exp(-g))
    elif c["act"] == "gelu_tanh":
        a = g / (1 + torch.exp(-math.sqrt(8 / math.pi) * (g + 0.044715 * g * g * g)))  # (1 + tanh x) / 2 = 1 / (1 + e^-2x)
    else:
        a = torch.relu(g) if c["act"] == "relu" else g
    y = (a * (t["x"] @ t["wu"])) @ t["wd"]
    y = y + t["x"] if c["res"] else y
    if c["dir"] == "fwd":
        return y
    grads = torch.autograd.grad(y, [t[k] for k in names], s["dy"].double())
    return dict(zip(("dx", "dwg", "dwu", "dwd"), grads))


def exact(case, seed):
    op = case["op"]
    if op == "ffn" and case["n"] * case["d"] * case["f"] * (18 if case["dir"] == "bwd" else 6) > 8e12:
        return None  # products in 64 bits run at about a TFLOP/s
    s = prepare(case, seed)
    if op == "qkrot":
        return _exact_qkrot(s, case)
    if op == "ffn":
        return _exact_ffn(s, case)
    if op == "decay":
        return _exact_decay(s, case)
    one = {x: s[x][:, None] for x in "qkv"}
    out = _exact_decay({**s, **one, "lens": s["live"], "s0": s["state"]}, case)
    return {"o": out["o"][:, 0], "state": out["state"]}
