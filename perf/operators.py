"""Measured cases of the operators of a fine-tuning step around the filtered convolution: layer norm (forward, backward
with the reduction of the weight's gradient), the Newton-Schulz orthogonalisation of an update, and the Muon step on a
list of layers of one shape.

With `own` false, run() computes an operator from elementary torch operations in 32 bits, rounded once at the end; with
`own` true it makes the calls of this package.  Sizes are those of the package's own workloads (96/576-channel inverted
residual block on 28 x 28 maps, 512-channel stages, 3x3 layers of 256 channels), or powers of two and odd sizes.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_ABC = (3.4445, -4.7750, 2.0315)        # quintic Newton-Schulz coefficients, five steps
_NS_EPS = 1e-7
_LN_EPS = 1e-5
_MOMENTUM, _DECAY = 0.95, 0.01


def _ln(name, way, n, c, h, w, layout, dtype, param="f32"):
    return {"name": name, "op": "layer_norm", "way": way, "n": n, "c": c, "h": h, "w": w, "layout": layout, "dtype": dtype,
            "param": param}


def _ns(name, batch, rows, cols, dtype, out):
    return {"name": name, "op": "newton_schulz", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype, "out": out}


def _muon(name, count, rows, cols, taps, weight):
    return {"name": name, "op": "muon", "count": count, "rows": rows, "cols": cols, "taps": taps, "weight": weight}


def listed():
    return [
        # a handful of rows: the head's norm of a small batch, or of one token; latency is all there is
        _ln("ln_fwd_8x768_bf16", "forward", 8, 768, 1, 1, "nhwc", "bf16"),
        # the block's expanded map, channels last: rows of 576
        _ln("ln_fwd_nhwc_576_28x28_f32", "forward", 128, 576, 28, 28, "nhwc", "f32"),
        # the same kind of map as the convolutions hold it by default: channels are planes apart, planes of odd size
        _ln("ln_fwd_nchw_96_55x55_bf16", "forward", 64, 96, 55, 55, "nchw", "bf16", "bf16"),
        # rows of an odd length: no row but the first starts on a vector boundary
        _ln("ln_bwd_4099x1001_f32", "backward", 4099, 1001, 1, 1, "nhwc", "f32"),
        # wide rows, as an MLP or a large head has them
        _ln("ln_bwd_8192x4096_bf16", "backward", 8192, 4096, 1, 1, "nhwc", "bf16"),
        # the stage of 512 channels on 16 x 16 maps, channels first
        _ln("ln_bwd_nchw_512_16x16_f32", "backward", 256, 512, 16, 16, "nchw", "f32"),
        # the 1x1 projections of a block: one small matrix, latency counts
        _ns("ns_1x96x576_f32_bf16", 1, 96, 576, "f32", "bf16"),
        # a stage's projections at once, tall, results in 32 bits
        _ns("ns_4x2048x512_f32_f32", 4, 2048, 512, "f32", "f32"),
        # the largest square matrix that one GPU's layer has in practice
        _ns("ns_1x4096x4096_bf16_bf16", 1, 4096, 4096, "bf16", "bf16"),
        # the 3x3 layers of a 256-channel stage with filtered gradients: all taps of g_W are equal
        _muon("muon_6x256x256x9_f32", 6, 256, 256, 9, "f32"),
        # a head with exact gradients and an odd number of classes
        _muon("muon_1x1001x2048_f32", 1, 1001, 2048, 1, "f32"),
        # the small projections of many blocks in one call
        _muon("muon_12x576x96_bf16", 12, 576, 96, 1, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("forward", "backward", "newton_schulz", "muon"))
    if op in ("forward", "backward"):
        total = _log(rng, 1 << 10, 1 << 26)
        dtype, param = rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16"))
        if rng.random() < 0.5:
            c = min(total, _log(rng, 16, 8192))
            return _ln("drawn", op, max(1, total // c), c, 1, 1, "nhwc", dtype, param)
        c = _log(rng, 8, 1024)
        side = max(1, min(_log(rng, 1, 112), int(math.sqrt(total / c)) or 1))
        w = max(1, side + rng.choice((-1, 0, 0, 1)))
        n = max(1, total // (c * side * w))
        return _ln("drawn", op, n, c, side, w, rng.choice(("nchw", "nchw", "nhwc")), dtype, param)
    most = 5 * 6.0 * 4096.0 ** 3
    if op == "newton_schulz":
        rows, cols, batch = _log(rng, 8, 4096), _log(rng, 8, 4096), _log(rng, 1, 12)
        m, n = min(rows, cols), max(rows, cols)
        out = rng.choice(("f32", "bf16", "bf16"))
        while batch > 1 and 5.0 * batch * (4.0 * m * m * n + 2.0 * m ** 3) > most / 3:
            batch -= 1
        return _ns("drawn", batch, rows, cols, rng.choice(("f32", "bf16")), out)
    rows, cols = _log(rng, 8, 1536), _log(rng, 8, 1536)
    taps = rng.choice((1, 1, 9, 9, 25)) if max(rows, cols) <= 512 else 1
    return _muon("drawn", _log(rng, 1, 12), rows, cols, taps, rng.choice(("f32", "f32", "bf16")))


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _gradient(g, batch, rows, cols):
    """A few strong directions that fall off, and noise: what weight gradients look like."""
    k = max(1, min(rows, cols) // 4)
    s = torch.arange(1, k + 1, device="cuda", dtype=torch.float32).rsqrt()
    low = (_randn(g, batch, rows, k) * s) @ _randn(g, batch, k, cols)
    return (low + _randn(g, batch, rows, cols)) * 1e-3


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "layer_norm":
        n, c, h, w = case["n"], case["c"], case["h"], case["w"]
        dt, pt = _DT[case["dtype"]], _DT[case["param"]]
        shape, ax = ((n, c, h, w), 1) if case["layout"] == "nchw" else ((n, h, w, c), 3)
        per_channel = [1, 1, 1, 1]
        per_channel[ax] = c
        # channels differ in scale and offset, a few of them strongly
        scale = (0.5 + torch.rand(c, generator=g, device="cuda") * (1 + 9 * (torch.rand(c, generator=g, device="cuda") < 0.01)))
        x = (_randn(g, *shape) * scale.view(per_channel) + 0.5 * _randn(g, c).view(per_channel)).to(dt)
        s = {"case": case, "ax": ax, "x": x, "gamma": (1 + 0.2 * _randn(g, c)).to(pt), "beta": (0.1 * _randn(g, c)).to(pt),
             "mean": torch.empty(n * h * w, device="cuda"), "rstd": torch.empty(n * h * w, device="cuda")}
        if case["way"] == "forward":
            s["y"] = torch.empty_like(x)
        else:
            s["gy"] = (1e-2 * _randn(g, *shape)).to(dt)
            x32 = x.float()
            s["mean"].copy_(x32.mean(ax).reshape(-1))
            s["rstd"].copy_((x32.var(ax, unbiased=False) + _LN_EPS).rsqrt().reshape(-1))
            s["gx"] = torch.empty_like(x)
            s["ggamma"], s["gbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        return s
    if case["op"] == "newton_schulz":
        G = _gradient(g, case["batch"], case["rows"], case["cols"]).to(_DT[case["dtype"]])
        return {"case": case, "G": G, "O": torch.empty(G.shape, dtype=_DT[case["out"]], device="cuda")}
    count, rows, cols, taps = case["count"], case["rows"], case["cols"], case["taps"]
    wt = _DT[case["weight"]]
    grad = _gradient(g, count, rows, cols)[..., None].expand(count, rows, cols, taps)      # filtered g_W: equal taps
    weight = (_randn(g, count, rows, cols, taps) * math.sqrt(2.0 / (cols * taps))).to(wt)
    buf = _gradient(g, count, rows, cols)
    lists = {"grad": [t.contiguous() for t in grad], "weight": [t.clone() for t in weight], "buf": [t.clone() for t in buf]}
    return {"case": case, "lr": 1e-3 if case["weight"] == "f32" else 2e-2, "scale": 0.2 * math.sqrt(max(rows, cols * taps)),
            **lists, "weight_out": [torch.empty_like(t) for t in lists["weight"]],
            "buf_out": [torch.empty_like(t) for t in lists["buf"]]}


# ---- the plain forms --------------------------------------------------------------------------------

def _plain_layer_norm(s):
    case, ax = s["case"], s["ax"]
    per_channel = [1, 1, 1, 1]
    per_channel[ax] = case["c"]
    rest = [d for d in range(4) if d != ax]
    x, gamma = s["x"].float(), s["gamma"].float().view(per_channel)
    if case["way"] == "forward":
        mean = x.mean(ax, keepdim=True)
        xc = x - mean
        rstd = 1.0 / torch.sqrt((xc * xc).mean(ax, keepdim=True) + _LN_EPS)
        y = xc * rstd * gamma + s["beta"].float().view(per_channel)
        return {"y": y.to(s["x"].dtype), "mean": mean.reshape(-1), "rstd": rstd.reshape(-1)}
    gy = s["gy"].float()
    rows = [d if i != ax else 1 for i, d in enumerate(x.shape)]
    rstd = s["rstd"].view(rows)
    xh = (x - s["mean"].view(rows)) * rstd
    h = gy * gamma
    gx = rstd * (h - h.mean(ax, keepdim=True) - xh * (h * xh).mean(ax, keepdim=True))
    return {"gx": gx.to(s["x"].dtype), "ggamma": (gy * xh).sum(rest), "gbeta": gy.sum(rest)}


def _quintic(X):
    a, b, c = _ABC
    A = X @ X.mT
    return a * X + (b * A + c * (A @ A)) @ X


def _plain_newton_schulz(G, eps=_NS_EPS):
    G = G.float()
    X = G if G.shape[-2] <= G.shape[-1] else G.mT
    X = X / (torch.sqrt((X * X).sum((-2, -1), keepdim=True)) + eps)
    X = _quintic(_quintic(_quintic(_quintic(_quintic(X)))))
    return X if G.shape[-2] <= G.shape[-1] else X.mT


def _plain_muon(s):
    taps = s["case"]["taps"]
    G = torch.stack(s["grad"])
    g = G[..., 0].float()
    buf = _MOMENTUM * torch.stack(s["buf"]) + (1 - _MOMENTUM) * g
    u = (1 - _MOMENTUM) * g + _MOMENTUM * buf
    # the flattened [rows, cols taps] matrix is u (x) 1: its norm and singular values are sqrt(taps) times those of u
    O = _plain_newton_schulz(u, _NS_EPS / math.sqrt(taps))[..., None] / math.sqrt(taps)
    W = torch.stack(s["weight"])
    new = (1 - s["lr"] * _DECAY) * W.float() - s["lr"] * s["scale"] * O
    return {"weight": list(new.to(W.dtype).unbind(0)), "buf": list(buf.unbind(0))}


# ---- the package's calls ----------------------------------------------------------------------------

def _own(s):
    import paper_2301_00330_b200 as gf

    case = s["case"]
    if case["op"] == "layer_norm":
        desc = s.get("desc")
        if desc is None:      # a program makes its descriptors and workspaces on its first pass
            desc = s["desc"] = gf.make_norm_desc(case["n"], case["c"], case["h"], case["w"], dtype=_DT[case["dtype"]],
                                                 param_dtype=_DT[case["param"]], eps=_LN_EPS,
                                                 layout=gf.GF_NCHW if case["layout"] == "nchw" else gf.GF_NHWC)
            if case["way"] == "backward":
                s["ws"] = torch.empty(gf.gf_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        if case["way"] == "forward":
            gf.gf_layer_norm_forward(desc, s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        gf.gf_layer_norm_backward(desc, s["gy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["gx"], s["ggamma"], s["gbeta"],
                                  s["ws"])
        return {"gx": s["gx"], "ggamma": s["ggamma"], "gbeta": s["gbeta"]}
    if case["op"] == "newton_schulz":
        desc = s.get("desc")
        if desc is None:
            desc = s["desc"] = gf.make_ns_desc(case["batch"], case["rows"], case["cols"], in_dtype=_DT[case["dtype"]],
                                               out_dtype=_DT[case["out"]], eps=_NS_EPS,
                                               precision=gf.GF_NS_F32 if case["out"] == "f32" else gf.GF_NS_F16)
            s["ws"] = torch.empty(gf.gf_newton_schulz_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        gf.gf_newton_schulz(desc, s["G"], s["O"], s["ws"])
        return s["O"]
    desc = s.get("desc")
    if desc is None:
        desc = s["desc"] = gf.make_muon_desc(case["count"], case["rows"], case["cols"], case["taps"], grad_dtype=torch.float32,
                                             weight_dtype=_DT[case["weight"]], eps=_NS_EPS,
                                             precision=gf.GF_NS_F32 if case["weight"] == "f32" else gf.GF_NS_F16,
                                             momentum=_MOMENTUM, nesterov=True, lr=s["lr"], weight_decay=_DECAY,
                                             scale=s["scale"])
        s["ws"] = torch.empty(gf.gf_muon_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    gf.gf_muon_step(desc, s["grad"], s["buf"], s["weight"], s["buf_out"], s["weight_out"], s["ws"])
    return {"weight": s["weight_out"], "buf": s["buf_out"]}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "layer_norm":
        return _plain_layer_norm(state)
    if op == "newton_schulz":
        return _plain_newton_schulz(state["G"]).to(state["O"].dtype)
    return _plain_muon(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------

def _ns_flops(rows, cols, steps=5):
    m, n = min(rows, cols), max(rows, cols)
    return steps * (float(m) * (m + 1) * n + float(m) * m * (m + 1) + 2.0 * m * m * n)     # A and A A are symmetric


def work(case):
    e = {"f32": 4, "bf16": 2}
    if case["op"] == "layer_norm":
        rows, c, b, p = case["n"] * case["h"] * case["w"], case["c"], e[case["dtype"]], e[case["param"]]
        if case["way"] == "forward":
            return {"bytes": 2 * rows * c * b + 8 * rows + 2 * c * p, "flops": 8.0 * rows * c}
        return {"bytes": 3 * rows * c * b + 8 * rows + c * (p + 8), "flops": 14.0 * rows * c}
    if case["op"] == "newton_schulz":
        mn = case["batch"] * case["rows"] * case["cols"]
        return {"bytes": mn * (e[case["dtype"]] + e[case["out"]]), "flops": case["batch"] * _ns_flops(case["rows"], case["cols"])}
    mn = case["count"] * case["rows"] * case["cols"]
    return {"bytes": mn * (4 + 8 + 2 * case["taps"] * e[case["weight"]]),
            "flops": case["count"] * _ns_flops(case["rows"], case["cols"])}


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def _exact_ns(u):
    """All factors of the iteration are polynomials in S = X X^T and commute: P = B_K ... B_1, result P X.  In 64 bits."""
    X = u if u.shape[-2] <= u.shape[-1] else u.transpose(-2, -1)
    X = X / (torch.linalg.vector_norm(X, dim=(-2, -1), keepdim=True) + _NS_EPS)
    S = X @ X.transpose(-2, -1)
    eye = torch.eye(S.shape[-1], dtype=S.dtype, device=S.device)
    P = eye.expand_as(S)
    for _ in range(5):
        B = _ABC[0] * eye + _ABC[1] * S + _ABC[2] * torch.matmul(S, S)
        P, S = B @ P, B @ S @ B
    X = P @ X
    return X if u.shape[-2] <= u.shape[-1] else X.transpose(-2, -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "layer_norm":
        ax = s["ax"]
        to_rows = (0, 2, 3, 1) if ax == 1 else (0, 1, 2, 3)
        back = (0, 3, 1, 2) if ax == 1 else (0, 1, 2, 3)
        x = s["x"].double().permute(to_rows)
        gamma, beta = s["gamma"].double(), s["beta"].double()
        if case["way"] == "forward":
            var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
            rstd = (var + _LN_EPS) ** -0.5
            y = (x - mean) * (rstd * gamma) + beta
            return {"y": y.permute(back).contiguous(), "mean": mean.reshape(-1), "rstd": rstd.reshape(-1)}
        gy = s["gy"].double().permute(to_rows)
        mean, rstd = s["mean"].double().view(x.shape[:3] + (1,)), s["rstd"].double().view(x.shape[:3] + (1,))
        xh = (x - mean) * rstd
        c1 = torch.einsum("nhwc,nhwc,c->nhw", gy, xh, gamma)[..., None] / case["c"]
        c2 = torch.einsum("nhwc,c->nhw", gy, gamma)[..., None] / case["c"]
        gx = (gy * gamma - c2 - xh * c1) * rstd
        return {"gx": gx.permute(back).contiguous(), "ggamma": torch.einsum("nhwc,nhwc->c", gy, xh), "gbeta": gy.sum((0, 1, 2))}
    if case["op"] == "newton_schulz":
        return _exact_ns(s["G"].double())
    # each layer from its whole flattened gradient [rows, cols taps], as the step is defined
    count, rows, cols, taps = case["count"], case["rows"], case["cols"], case["taps"]
    g = torch.stack([t.double() for t in s["grad"]])
    b0 = torch.stack([t.double() for t in s["buf"]])
    buf = b0 + (1 - _MOMENTUM) * (g[..., 0] - b0)
    u = (g + _MOMENTUM * (buf[..., None] - g)).reshape(count, rows, cols * taps)
    O = _exact_ns(u).reshape(count, rows, cols, taps)
    W = torch.stack([t.double() for t in s["weight"]])
    W = W - s["lr"] * (_DECAY * W + s["scale"] * O)
    return {"weight": list(W.unbind(0)), "buf": list(buf.unbind(0))}
