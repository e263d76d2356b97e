"""Measured cases of the operators of a residual block whose layers are frozen in 8 bits: dropout from a counter with the
residual's addition, root-mean-square norm of that sum with results in 16, 32 or 8 bits and its backward pass, and the products
of 8-bit rows with 8-bit weights (forward, and the gradient of the input).

With `own` false, run() computes an operator from elementary torch operations in 32 bits, rounded once at the end; with
`own` true it makes the calls of this package.  Sizes are those of the package's own workloads (576-channel maps of
128 x 28 x 28 pixels, 512 -> 2048 channels on 256 x 16 x 16, a head of 1001 classes), or powers of two and odd sizes.

8-bit matrices are e4m3 codes in rows of round_up(cols, 16) bytes, with a scale for each 128 columns of a row, stored
[ceil(cols / 128)][round_up(rows, 4)], or for each 128 x 128 block of a weight.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5
_TOP = 448.0                 # largest e4m3 value
_TINY = 2.0 ** -126          # smallest scale


def _drop(name, way, rows, cols, dtype, p):
    return {"name": name, "op": "dropout", "way": way, "rows": rows, "cols": cols, "dtype": dtype, "p": p}


def _rms(name, way, rows, cols, dtype, residual, p):
    return {"name": name, "op": "rms_norm", "way": way, "rows": rows, "cols": cols, "dtype": dtype, "residual": residual, "p": p}


def _mm(name, way, m, n, k, source, out, bias):
    return {"name": name, "op": "fp8", "way": way, "m": m, "n": n, "k": k, "source": source, "out": out, "bias": bias}


def listed():
    return [
        # the features of a small batch in front of a head: latency is all there is
        _drop("drop_fwd_8x768_bf16", "forward", 8, 768, "bf16", 0.1),
        # the branch of a block on 576-channel maps, channels last, added to its skip connection
        _drop("drop_fwd_100352x576_bf16", "forward", 100352, 576, "bf16", 0.1),
        # a gradient on its way back, rows of odd length
        _drop("drop_bwd_4099x1001_f32", "backward", 4099, 1001, "f32", 0.5),
        # a few rows on their way into a frozen 8-bit layer
        _rms("rms_fwd8_8x768_bf16", "forward8", 8, 768, "bf16", "bf16", 0.0),
        # the block's maps, a dropped branch added in the same pass
        _rms("rms_fwd_100352x576_bf16", "forward", 100352, 576, "bf16", "bf16", 0.1),
        # wide rows with the residual kept in 32 bits, normed straight into 8 bits
        _rms("rms_fwd8_16384x2048_bf16", "forward8", 16384, 2048, "bf16", "f32", 0.0),
        # rows of an odd length: no row but the first starts on a vector boundary
        _rms("rms_bwd_4099x1001_f32", "backward", 4099, 1001, "f32", "f32", 0.1),
        # wide rows, as an MLP has them
        _rms("rms_bwd_8192x4096_bf16", "backward", 8192, 4096, "bf16", "bf16", 0.0),
        # a few rows through a large frozen layer, straight from the norm's 8 bits: the weight's bytes count
        _mm("mm_fwd_8x4096x4096_bf16", "forward", 8, 4096, 4096, "codes", "bf16", False),
        # a head with an odd number of classes on an odd number of rows, logits in 32 bits
        _mm("mm_fwd_4099x1001x576_f32", "forward", 4099, 1001, 576, "codes", "f32", True),
        # a frozen 1x1 layer 512 -> 2048 on 256 x 16 x 16 maps: its 16-bit input is quantised and multiplied
        _mm("lin_fwd_65536x2048x512_bf16", "forward", 65536, 2048, 512, "bf16", "bf16", True),
        # the gradient through a large frozen layer: 16-bit g_y quantised, times the weight as it is stored
        _mm("lin_gx_4096x8192x4096_bf16", "gradient", 4096, 8192, 4096, "bf16", "bf16", False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("dropout", "rms_norm", "rms_norm", "fp8", "fp8"))
    if op == "dropout":
        total, cols = _log(rng, 1 << 10, 1 << 25), _log(rng, 16, 8192)
        cols = min(total, cols)
        return _drop("drawn", rng.choice(("forward", "backward")), max(1, total // cols), cols, rng.choice(("f32", "bf16")),
                     round(rng.uniform(0.02, 0.6), 3))
    if op == "rms_norm":
        total, cols = _log(rng, 1 << 10, 1 << 25), _log(rng, 16, 8192)
        cols = min(total, cols)
        if rng.random() < 0.5:
            cols = -(-cols // 16) * 16
        dtype = rng.choice(("f32", "bf16"))
        residual = rng.choice(("f32", "bf16")) if dtype == "bf16" else "f32"
        return _rms("drawn", rng.choice(("forward", "forward8", "backward")), max(1, total // cols), cols, dtype, residual,
                    rng.choice((0.0, 0.0, 0.1, 0.25)))
    m, n, k = _log(rng, 1, 65536), _log(rng, 64, 8192), _log(rng, 64, 8192)
    if rng.random() < 0.5:
        n, k = -(-n // 64) * 64, -(-k // 64) * 64
    while m * n * k > 1.2e11 or m * max(n, k) > 1.2e8:
        m = max(1, m // 2)
    way = rng.choice(("forward", "forward", "gradient"))
    return _mm("drawn", way, m, n, k, rng.choice(("codes", "f32", "bf16")), rng.choice(("f32", "bf16", "bf16")),
               way == "forward" and rng.random() < 0.5)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _channels(g, cols):
    """Channels differ in scale, a few of them strongly."""
    return 0.5 + torch.rand(cols, generator=g, device="cuda") * (1 + 9 * (torch.rand(cols, generator=g, device="cuda") < 0.01))


def _seed_words(seed):
    return torch.tensor([(seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), seed], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "dropout":
        shape, dt = (case["rows"], case["cols"]), _DT[case["dtype"]]
        s = {"case": case, "seed": _seed_words(seed), "y": torch.empty(shape, dtype=dt, device="cuda")}
        if case["way"] == "forward":
            s["x"], s["res"] = _randn(g, *shape).to(dt), (2 * _randn(g, *shape)).to(dt)
        else:
            s["x"] = (1e-2 * _randn(g, *shape)).to(dt)
        return s
    if case["op"] == "rms_norm":
        rows, cols, dt, rt = case["rows"], case["cols"], _DT[case["dtype"]], _DT[case["residual"]]
        s = {"case": case, "seed": _seed_words(seed), "gamma": 1 + 0.2 * _randn(g, cols)}
        h = _randn(g, rows, cols) * _channels(g, cols) + 0.3 * _randn(g, cols)
        if case["way"] == "backward":
            s["h"] = h.to(rt)
            s["rstd"] = (s["h"].float().square().mean(1) + _EPS).rsqrt()
            s["gy"], s["gh"] = (1e-2 * _randn(g, rows, cols)).to(dt), (1e-2 * _randn(g, rows, cols)).to(rt)
            s["gres"] = torch.empty_like(s["h"])
            s["gx"] = None if case["p"] == 0 and dt == rt else torch.empty_like(s["gy"])
            s["ggamma"] = torch.empty(cols, device="cuda")
            return s
        s["res"], s["x"] = h.to(rt), (0.5 * _randn(g, rows, cols)).to(dt)
        s["h"], s["rstd"] = torch.empty_like(s["res"]), torch.empty(rows, device="cuda")
        if case["way"] == "forward":
            s["y"] = torch.empty_like(s["x"])
        else:
            s["codes"], s["scales"] = _room(rows, cols)
        return s
    m, n, k = case["m"], case["n"], case["k"]
    w, wq = _blocks8(_randn(g, n, k) * math.sqrt(1.0 / k) * (0.5 + torch.rand(n, 1, generator=g, device="cuda")))
    inner, outer = (k, n) if case["way"] == "forward" else (n, k)
    x = _randn(g, m, inner) * _channels(g, inner) * (1.0 if case["way"] == "forward" else 1e-2)
    s = {"case": case, "w": w, "w_scales": wq, "bias": _randn(g, outer) if case["bias"] else None,
         "out": torch.empty((m, outer), dtype=_DT[case["out"]], device="cuda")}
    if case["source"] == "codes":
        s["a"], s["a_scales"] = _rows8(x)
    else:
        s["x"] = x.to(_DT[case["source"]])
        s["a"], s["a_scales"] = _room(m, inner)
    return s


# ---- 8-bit matrices as they are stored ------------------------------------------------------------------

def _up(n, to):
    return -(-n // to) * to


def _room(rows, cols):
    return (torch.empty((rows, _up(cols, 16)), dtype=torch.float8_e4m3fn, device="cuda"),
            torch.empty((_up(cols, 128) // 128, _up(rows, 4)), device="cuda"))


def _padded(x, rows, cols):
    p = torch.zeros((rows, cols), dtype=torch.float32, device=x.device)
    p[:x.shape[0], :x.shape[1]] = x
    return p


def _row_groups(x):
    """Codes as float32 [rows, cols] and scales [groups, rows] of fp32 rows."""
    rows, cols = x.shape
    t = _padded(x, rows, _up(cols, 128)).view(rows, -1, 128)
    scale = (t.abs().amax(2) / _TOP).clamp_min(_TINY)
    q = (t / scale[..., None]).to(torch.float8_e4m3fn)
    return q.view(rows, -1)[:, :cols], scale.t()


def _rows8(x):
    rows, cols = x.shape
    q, scale = _row_groups(x)
    codes = torch.zeros((rows, _up(cols, 16)), dtype=torch.uint8, device=x.device)
    codes[:, :cols] = q.contiguous().view(torch.uint8)
    return codes.view(torch.float8_e4m3fn), _padded(scale, scale.shape[0], _up(rows, 4))


def _blocks8(w):
    n, k = w.shape
    t = _padded(w, _up(n, 128), _up(k, 128)).view(_up(n, 128) // 128, 128, -1, 128)
    scale = (t.abs().amax((1, 3)) / _TOP).clamp_min(_TINY)
    q = (t / scale[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(_up(n, 128), -1)
    return q[:n, :_up(k, 16)].contiguous().view(torch.float8_e4m3fn), scale.contiguous()


# ---- the plain forms --------------------------------------------------------------------------------------

def _mul_hi_lo(m, a):
    """High and low halves of the 64-bit product of a 32-bit constant and 32-bit values held in int64."""
    low = (a & 0xFFFF) * m
    t = (a >> 16) * m + (low >> 16)
    return t >> 16, ((t & 0xFFFF) << 16) | (low & 0xFFFF)


def _philox_round(c, k):
    h0, l0 = _mul_hi_lo(0xD2511F53, c[0])
    h1, l1 = _mul_hi_lo(0xCD9E8D57, c[2])
    return [h1 ^ c[1] ^ k[0], l1, h0 ^ c[3] ^ k[1], l0], [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]


def _keep(s):
    """Truth values [rows, cols]: element i has 16 bits of its own, word i % 8 / 2 of block i / 8, the low half first."""
    case = s["case"]
    n = case["rows"] * case["cols"]
    block = torch.arange(-(-n // 8), device="cuda")
    key, offset = s["seed"][0], s["seed"][1]
    zero = torch.zeros_like(block)
    c = [block & 0xFFFFFFFF, block >> 32, zero + (offset & 0xFFFFFFFF), zero + ((offset >> 32) & 0xFFFFFFFF)]
    k = [key & 0xFFFFFFFF, (key >> 32) & 0xFFFFFFFF]
    c, k = _philox_round(*_philox_round(*_philox_round(*_philox_round(*_philox_round(c, k)))))
    c, k = _philox_round(*_philox_round(*_philox_round(*_philox_round(*_philox_round(c, k)))))
    w = torch.stack(c, 1)
    bits = torch.stack((w & 0xFFFF, w >> 16), 2).reshape(-1)[:n]
    return (bits >= _threshold(case["p"])).view(case["rows"], case["cols"])


def _threshold(p):
    return int(round(p * 65536.0))


def _dropped(s, x):
    t = _threshold(s["case"]["p"])
    if t == 0:
        return x
    return torch.where(_keep(s), x * (65536.0 / (65536 - t)), torch.zeros_like(x))


def _plain_rms(s):
    case = s["case"]
    dt, rt = _DT[case["dtype"]], _DT[case["residual"]]
    if case["way"] == "backward":
        h, rstd, gy = s["h"].float(), s["rstd"][:, None], s["gy"].float()
        xh = h * rstd
        hg = gy * s["gamma"]
        d = rstd * (hg - xh * (hg * xh).mean(1, keepdim=True)) + s["gh"].float()
        out = {"gres": d.to(rt), "ggamma": (gy * xh).sum(0)}
        return out if s["gx"] is None else {**out, "gx": _dropped(s, d).to(dt)}
    h = (s["res"].float() + _dropped(s, s["x"].float())).to(rt)
    hf = h.float()
    rstd = 1.0 / torch.sqrt((hf * hf).mean(1, keepdim=True) + _EPS)
    y = hf * rstd * s["gamma"]
    out = {"h": h, "rstd": rstd[:, 0]}
    if case["way"] == "forward":
        return {**out, "y": y.to(dt)}
    q, scale = _row_groups(y)
    return {**out, "codes": q, "scales": scale}


def _plain_product(s):
    case = s["case"]
    inner = case["k"] if case["way"] == "forward" else case["n"]
    if case["source"] == "codes":
        a, scale = s["a"][:, :inner].float(), s["a_scales"][:, :case["m"]]
    else:
        a, scale = _row_groups(s["x"].float())
        a = a.float()
    a = a * scale.t().repeat_interleave(128, 1)[:, :inner]
    n, k = case["n"], case["k"]
    w = s["w"][:, :k].float() * s["w_scales"].repeat_interleave(128, 0).repeat_interleave(128, 1)[:n, :k]
    out = a @ w.t() if case["way"] == "forward" else a @ w
    return (out if s["bias"] is None else out + s["bias"]).to(s["out"].dtype)


# ---- the package's calls ----------------------------------------------------------------------------

def _own(s):
    import paper_2301_00330_b200 as gf

    case = s["case"]
    desc = s.get("desc")
    if case["op"] == "dropout":
        if desc is None:      # a program makes its descriptors and workspaces on its first pass
            dt = _DT[case["dtype"]]
            desc = s["desc"] = gf.make_dropout_desc(case["rows"] * case["cols"], dtype=dt, p=case["p"])
        if case["way"] == "forward":
            gf.gf_dropout_forward(desc, s["x"], s["res"], s["seed"], s["y"])
        else:
            gf.gf_dropout_backward(desc, s["x"], s["seed"], s["y"])
        return s["y"]
    if case["op"] == "rms_norm":
        if desc is None:
            desc = s["desc"] = gf.make_rms_desc(case["rows"], case["cols"], dtype=_DT[case["dtype"]],
                                                residual_dtype=_DT[case["residual"]], eps=_EPS, p=case["p"])
            if case["way"] == "backward":
                s["ws"] = torch.empty(gf.gf_rms_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        seed = s["seed"] if case["p"] > 0 else None
        if case["way"] == "backward":
            gf.gf_rms_norm_backward(desc, s["gy"], s["gh"], s["h"], s["rstd"], s["gamma"], seed, s["gres"], s["gx"], s["ggamma"],
                                    s["ws"])
            out = {"gres": s["gres"], "ggamma": s["ggamma"]}
            return out if s["gx"] is None else {**out, "gx": s["gx"]}
        if case["way"] == "forward":
            gf.gf_rms_norm_forward(desc, s["x"], s["res"], seed, s["gamma"], s["h"], s["y"], s["rstd"])
            return {"h": s["h"], "rstd": s["rstd"], "y": s["y"]}
        gf.gf_rms_norm_forward_fp8(desc, s["x"], s["res"], seed, s["gamma"], s["h"], s["codes"], s["scales"], s["rstd"])
        return {"h": s["h"], "rstd": s["rstd"], "codes": s["codes"][:, :case["cols"]], "scales": s["scales"][:, :case["rows"]]}
    if desc is None:
        desc = s["desc"] = gf.make_fp8_matmul_desc(case["m"], case["n"], case["k"], transposed=case["way"] == "gradient",
                                                   out_dtype=_DT[case["out"]])
        if case["source"] != "codes":
            s["rows_desc"] = gf.make_fp8_desc(case["m"], s["x"].shape[1], dtype=_DT[case["source"]])
    if case["source"] != "codes":
        gf.gf_fp8_quantize_rows(s["rows_desc"], s["x"], s["a"], s["a_scales"])
    gf.gf_fp8_matmul(desc, s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], s["out"])
    return s["out"]


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "dropout":
        y = _dropped(state, state["x"].float())
        return (y if case["way"] == "backward" else state["res"].float() + y).to(state["y"].dtype)
    return _plain_rms(state) if case["op"] == "rms_norm" else _plain_product(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    e = {"f32": 4, "bf16": 2}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e[case["dtype"]] * (3 if case["way"] == "forward" else 2) + 16, "flops": 2.0 * n}
    if case["op"] == "rms_norm":
        rows, cols, b, r = case["rows"], case["cols"], e[case["dtype"]], e[case["residual"]]
        n = rows * cols
        if case["way"] == "backward":
            gx = 0 if case["p"] == 0 and b == r else b
            return {"bytes": n * (b + 3 * r + gx) + 4 * rows + 8 * cols, "flops": 10.0 * n}
        out = n * b if case["way"] == "forward" else n + 4 * rows * -(-cols // 128)
        return {"bytes": n * (b + 2 * r) + out + 4 * rows + 4 * cols, "flops": 6.0 * n}
    m, n, k = case["m"], case["n"], case["k"]
    inner, outer = (k, n) if case["way"] == "forward" else (n, k)
    groups = -(-inner // 128)
    read = m * (inner + 4 * groups) if case["source"] == "codes" else m * inner * e[case["source"]]
    weight = n * k + 4 * -(-n // 128) * -(-k // 128)
    return {"bytes": read + weight + m * outer * e[case["out"]] + (4 * outer if case["bias"] else 0), "flops": 2.0 * m * n * k}


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def _exact_keep(case, words):
    """Philox4x32 of ten rounds on unsigned 64-bit integers of the host."""
    n = case["rows"] * case["cols"]
    key, offset = (int(v) & 0xFFFFFFFFFFFFFFFF for v in words.tolist())
    block = np.arange(-(-n // 8), dtype=np.uint64)
    mask, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    x0, x1 = block & mask, block >> half
    x2, x3 = np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)
    k0, k1 = key & 0xFFFFFFFF, key >> 32
    for _ in range(10):
        p0, p1 = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (p1 >> half) ^ x1 ^ np.uint64(k0), p1 & mask, (p0 >> half) ^ x3 ^ np.uint64(k1), p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) % (1 << 32), (k1 + 0xBB67AE85) % (1 << 32)
    bits = np.stack((x0, x1, x2, x3), 1).astype(np.uint32).view(np.uint16).reshape(-1)[:n]
    return torch.from_numpy(bits.astype(np.int32) >= int(round(case["p"] * 65536.0))).cuda().view(case["rows"], case["cols"])


def _exact_dropped(s, x):
    t = int(round(s["case"]["p"] * 65536.0))
    return x * _exact_keep(s["case"], s["seed"]) * (65536.0 / (65536 - t)) if t else x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        y = _exact_dropped(s, s["x"].double())
        return y if case["way"] == "backward" else y + s["res"].double()
    if case["op"] == "rms_norm":
        gamma = s["gamma"].double()
        if case["way"] == "backward":
            h, r, gy = s["h"].double(), s["rstd"].double(), s["gy"].double()
            dot = torch.einsum("rc,rc,c->r", gy, h, gamma) / case["cols"]
            d = torch.einsum("r,rc,c->rc", r, gy, gamma) - h * (r ** 3 * dot)[:, None] + s["gh"].double()
            out = {"gres": d, "ggamma": torch.einsum("rc,rc,r->c", gy, h, r)}
            return out if s["gx"] is None else {**out, "gx": _exact_dropped(s, d)}
        h = s["res"].double() + _exact_dropped(s, s["x"].double())
        stored = h.to(_DT[case["residual"]]).double()            # the norm is that of the sum as it is kept
        rstd = (torch.linalg.vector_norm(stored, dim=1) ** 2 / case["cols"] + _EPS) ** -0.5
        y = stored * rstd[:, None] * gamma
        if case["way"] == "forward":
            return {"h": h, "rstd": rstd, "y": y}
        # codes: the values that are rounded to 8 bits
        parts = y.split(128, 1)
        scales = torch.stack([p.abs().amax(1) for p in parts]) / _TOP
        codes = torch.cat([p / t.clamp_min(_TINY)[:, None] for p, t in zip(parts, scales)], 1)
        return {"h": h, "rstd": rstd, "codes": codes, "scales": scales.clamp_min(_TINY)}
    m, n, k = case["m"], case["n"], case["k"]
    inner = k if case["way"] == "forward" else n
    if case["source"] == "codes":
        codes, scales = s["a"][:, :inner], s["a_scales"][:, :m]
    else:
        # a scale is a stored fp32 number, and so is the quotient that is rounded to a code
        x = s["x"].float()
        parts = x.split(128, 1)
        scales = torch.stack([(p.abs().amax(1) / _TOP).clamp_min(_TINY) for p in parts])
        codes = torch.cat([(p / t[:, None]).to(torch.float8_e4m3fn) for p, t in zip(parts, scales)], 1)
    out = torch.zeros((m, case["n"] if case["way"] == "forward" else k), dtype=torch.float64, device="cuda")
    w = s["w"][:, :k].double()
    for i in range(w.shape[0] // 128 + (w.shape[0] % 128 > 0)):
        for j in range(s["w_scales"].shape[1]):
            w[128 * i:128 * i + 128, 128 * j:128 * j + 128] *= s["w_scales"][i, j].double()
    for g in range(scales.shape[0]):                             # one group of 128 terms after the other
        at = slice(128 * g, min(128 * g + 128, inner))
        a = codes[:, at].double() * scales[g].double()[:, None]
        out += a @ (w[:, at].t() if case["way"] == "forward" else w[at])
    return out if s["bias"] is None else out + s["bias"].double()
