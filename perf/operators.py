"""Cases of the fused FP8 operators: the product with bias, activation and residual in its epilogue and its backward
pass, the gated feed-forward block and its backward pass, and the global gradient norm with clipping.

`run` computes them in their plain form (elementary torch operations in binary32 on the decoded codes, rounded once at
the end) or, where `own` is true, through the package's entry points.  FP8 results are returned as float8 views, that is
as the values the codes stand for.
"""
import math

import torch

own = False

DEV = "cuda"
FMAX = {"e4m3": 448.0, "e5m2": 57344.0}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
WIDE = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token through the down projection of the hidden-4096 layer, added to the residual stream (decoding)
        dict(name="epi_down_1", op="epilogue", tokens=1, d_in=16384, d_out=4096, act="none", bias=False, residual="bf16", pre=False,
             out="bf16", weight="kn", channel=False),
        # a small decoding batch through the up projection of a post-training quantized layer: per-channel weight scales, codes out
        dict(name="epi_up_37", op="epilogue", tokens=37, d_in=4096, d_out=16384, act="gelu", bias=True, residual="", pre=False,
             out="e4m3", weight="nk", channel=True),
        # a prompt of odd length through the widest down projection, fp32 residual stream
        dict(name="epi_down_1001", op="epilogue", tokens=1001, d_in=49152, d_out=12288, act="none", bias=True, residual="f32", pre=False,
             out="f32", weight="kn", channel=False),
        # training forward of the hidden-4096 up projection: the value before the activation is kept for the backward pass
        dict(name="epi_up_8192", op="epilogue", tokens=8192, d_in=4096, d_out=16384, act="gelu_tanh", bias=True, residual="", pre=True,
             out="e4m3", weight="kn", channel=False),
        # its backward pass: gradient through the activation to E5M2 codes, with the bias gradient
        dict(name="epi_bwd_8192", op="epilogue_backward", tokens=8192, d_out=16384, act="gelu_tanh", wide="bf16", out="e5m2"),
        # the same for a short odd batch of the hidden-12288 layer in fp32
        dict(name="epi_bwd_77", op="epilogue_backward", tokens=77, d_out=12289, act="gelu", wide="f32", out="e5m2"),
        # one token through the gated up projections (decoding)
        dict(name="gated_1", op="gated", tokens=1, d_in=4096, d_out=16384, act="silu", save=False, out="e4m3", weight="kn"),
        # training forward, both pre-products kept
        dict(name="gated_8192", op="gated", tokens=8192, d_in=4096, d_out=16384, act="silu", save=True, out="e4m3", weight="kn"),
        # training backward of the block's inner part: down-projection data gradient and the gate's derivative
        dict(name="gated_bwd_8192", op="gated_backward", tokens=8192, d_in=4096, d_out=16384, act="silu", out="e5m2", weight="kn", chain=False),
        # a short odd batch, on to the gradients of the input and of both up weights
        dict(name="gated_bwd_333", op="gated_backward", tokens=333, d_in=1024, d_out=4112, act="gelu_tanh", out="e5m2", weight="kn", chain=True),
        # biases and norm weights of 48 layers: many small gradients
        dict(name="clip_small", op="clip", count=288, big=16384, small=4096, inp="bf16", out="bf16"),
        # four layers' FFN weight gradients
        dict(name="clip_ffn", op="clip", count=12, big=4096 * 16384, small=4096 * 16384, inp="bf16", out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["epilogue", "epilogue_backward", "gated", "gated_backward", "clip"])
    while True:
        if op == "clip":
            c = dict(op=op, count=_log(rng, 1, 300), big=_log(rng, 64, 60_000_000), small=_log(rng, 1, 20000),
                     inp=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
            if c["count"] * max(c["big"], c["small"]) <= 12 * 4096 * 16384:
                return c
        elif op == "epilogue_backward":
            c = dict(op=op, tokens=_log(rng, 1, 8192), d_out=_log(rng, 48, 49152), act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                     wide=rng.choice(["bf16", "f32"]), out=rng.choice(["e5m2", "e4m3", "bf16"]))
            if c["tokens"] * c["d_out"] <= 8192 * 16384:
                return c
        else:
            c = dict(op=op, tokens=_log(rng, 1, 8192), d_in=_log(rng, 64, 16384), d_out=_log(rng, 64, 16384), weight=rng.choice(["kn", "nk"]))
            if op == "epilogue":
                c.update(act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), bias=rng.random() < 0.6,
                         residual=rng.choice(["", "bf16", "f32"]), pre=rng.random() < 0.3, out=rng.choice(["bf16", "bf16", "f32", "e4m3"]),
                         channel=rng.random() < 0.3)
            elif op == "gated":
                c.update(act=rng.choice(["silu", "gelu_tanh", "gelu"]), save=rng.random() < 0.5, out=rng.choice(["e4m3", "e4m3", "bf16"]))
            else:
                c.update(act=rng.choice(["silu", "gelu_tanh", "gelu"]), out=rng.choice(["e5m2", "e5m2", "bf16"]), weight="kn", chain=False)
            if c["tokens"] * c["d_in"] * c["d_out"] <= 8192 * 4096 * 16384:
                return c


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _pitch(cols, itemsize):
    """Row pitch in elements: the next multiple of 16 bytes."""
    unit = 16 // itemsize
    return -(-cols // unit) * unit


def _rows(rows, cols, dtype):
    """An uninitialised [rows, cols] matrix whose rows start on 16 bytes."""
    return torch.empty(rows, _pitch(cols, torch.empty(0, dtype=dtype).element_size()), dtype=dtype, device=DEV)[:, :cols]


def _put(values, dtype):
    m = _rows(values.shape[0], values.shape[1], dtype)
    m.copy_(values)
    return m


def _scalar(v):
    return torch.tensor([v], dtype=torch.float32, device=DEV)


def _codes(values, fmt, per_row=False):
    """FP8 codes of a matrix and its inverse scale (one, or one per row)."""
    amax = values.abs().amax(dim=1, keepdim=True) if per_row else values.abs().max().reshape(1, 1)
    scale = FMAX[fmt] / amax.clamp(min=1e-30)
    q = (values * scale).clamp(-FMAX[fmt], FMAX[fmt]).to(F8[fmt]).view(torch.uint8)
    return _put(q, torch.uint8), (1.0 / scale).reshape(-1).contiguous()


def _activations(g, rows, cols):
    x = torch.randn(rows, cols, generator=g, device=DEV)
    far = torch.rand(rows, cols, generator=g, device=DEV) < 0.001
    return torch.where(far, x.sign() * (20 + 80 * torch.rand(rows, cols, generator=g, device=DEV)), x)


def _gradients(g, rows, cols):
    """Student-t with 3 degrees of freedom, times 1e-4."""
    n = torch.randn(rows, cols, generator=g, device=DEV)
    s = sum(torch.randn(rows, cols, generator=g, device=DEV).square() for _ in range(3))
    return n * (1e-4 * math.sqrt(3.0)) / s.sqrt().clamp(min=1e-3)


def _weights(g, d_in, d_out, layout, fmt="e4m3", channel=False):
    """Weight codes stored [d_in, d_out] ("kn") or [d_out, d_in] ("nk"), standard deviation 0.02 at 4096 inputs."""
    w = torch.randn(d_out, d_in, generator=g, device=DEV) * (0.02 * math.sqrt(4096.0 / d_in))
    q, inv = _codes(w, fmt, per_row=channel)
    return (q if layout == "nk" else _put(q.t(), torch.uint8)), inv


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case=case)
    op = case["op"]
    if op == "epilogue":
        T, K, N = case["tokens"], case["d_in"], case["d_out"]
        s["x"], s["sx"] = _codes(_activations(g, T, K), "e4m3")
        s["w"], s["sw"] = _weights(g, K, N, case["weight"], channel=case["channel"])
        s["bias"] = torch.randn(N, generator=g, device=DEV).to(torch.bfloat16) if case["bias"] else None
        s["residual"] = _put(3 * torch.randn(T, N, generator=g, device=DEV), WIDE[case["residual"]]) if case["residual"] else None
        s["pre"] = _rows(T, N, torch.bfloat16) if case["pre"] else None
        s["d"] = _rows(T, N, WIDE.get(case["out"], torch.uint8))
        s["scale_d"], s["amax"] = _scalar(448.0 / 20.0), _scalar(0.0)
    elif op == "epilogue_backward":
        T, N = case["tokens"], case["d_out"]
        s["dy"] = _put(_gradients(g, T, N), WIDE[case["wide"]])
        s["pre"] = _put(2.5 * torch.randn(T, N, generator=g, device=DEV), WIDE[case["wide"]])
        s["dz"] = _rows(T, N, WIDE.get(case["out"], torch.uint8))
        s["dbias"] = torch.empty(N, dtype=torch.float32, device=DEV)
        s["scale_d"], s["amax"] = _scalar((57344.0 if case["out"] == "e5m2" else 448.0) / 0.02), _scalar(0.0)
    elif op == "gated":
        T, K, N = case["tokens"], case["d_in"], case["d_out"]
        s["x"], s["sx"] = _codes(_activations(g, T, K), "e4m3")
        s["wg"], s["sg"] = _weights(g, K, N, case["weight"])
        s["wu"], s["su"] = _weights(g, K, N, case["weight"])
        s["gate"], s["up"] = (_rows(T, N, torch.bfloat16), _rows(T, N, torch.bfloat16)) if case["save"] else (None, None)
        s["h"] = _rows(T, N, WIDE.get(case["out"], torch.uint8))
        s["scale_d"], s["amax"] = _scalar(448.0 / 200.0), _scalar(0.0)
    elif op == "gated_backward":
        T, K, N = case["tokens"], case["d_in"], case["d_out"]
        s["dy"], s["sy"] = _codes(_gradients(g, T, K), "e5m2")
        s["wd"], s["sd"] = _weights(g, N, K, case["weight"])
        s["gate"] = _put(2.5 * torch.randn(T, N, generator=g, device=DEV), torch.bfloat16)
        s["up"] = _put(2.5 * torch.randn(T, N, generator=g, device=DEV), torch.bfloat16)
        # the two gradients side by side: one tensor [tokens, 2 d_out] with one scale, as the following products read it
        wide = _pitch(N, 1) if case["out"] == "e5m2" else _pitch(N, 2)
        s["dgu"] = torch.zeros(T, 2 * wide, dtype=WIDE.get(case["out"], torch.uint8), device=DEV)
        s["dg"], s["du"] = s["dgu"][:, :N], s["dgu"][:, wide:wide + N]
        s["scale_d"], s["amax"] = _scalar(57344.0 / 0.05), _scalar(0.0)
        if case["chain"]:
            s["x"], s["sx"] = _codes(_activations(g, T, K), "e4m3")
            s["wgu"], s["sgu"] = _weights(g, K, 2 * N, "kn")
            s["inv_d"] = 1.0 / s["scale_d"]
            s["dx"], s["dw"] = _rows(T, K, torch.bfloat16), _rows(K, 2 * N, torch.bfloat16)
    else:
        n = [case["big"] if i % 2 == 0 else case["small"] for i in range(case["count"])]
        s["grads"] = [(torch.randn(k, generator=g, device=DEV) * (1e-4 * (1 + i % 5))).to(WIDE[case["inp"]]) for i, k in enumerate(n)]
        # the clipped gradients lie in one buffer, as an optimiser that walks a flat state keeps them; each starts on 16 bytes
        room = [_pitch(k, 2 if case["out"] == "bf16" else 4) for k in n]
        s["flat"] = torch.zeros(sum(room), dtype=WIDE[case["out"]], device=DEV)
        s["clipped"] = [t[:k] for t, k in zip(s["flat"].split(room), n)]
        s["norm"] = _scalar(0.0)
        # half of the expected norm, so that clipping takes place
        s["max_norm"] = 0.5e-4 * math.sqrt(sum(k * (1 + i % 5) ** 2 for i, k in enumerate(n)))
        if own:
            from paper_2209_05433_b200 import api
            s["plan"] = api.ClipPlan(s["grads"], s["clipped"])
    return s


# ---- the package's operators ----------------------------------------------------------------------------------------

def _own(s):
    from paper_2209_05433_b200 import api
    c = s["case"]
    act = {"none": api.ACT_NONE, "relu": api.ACT_RELU, "gelu": api.ACT_GELU, "gelu_tanh": api.ACT_GELU_TANH, "silu": api.ACT_SILU}
    fmt = {"e4m3": api.E4M3, "e5m2": api.E5M2}.get(c.get("out"))
    view = F8.get(c.get("out"))
    layout = api.MAJOR_MN if c.get("weight") == "kn" else api.MAJOR_K
    if c["op"] == "epilogue":
        codes = fmt is not None
        api.fp8_gemm_epilogue(s["x"], api.E4M3, api.MAJOR_K, s["w"], api.E4M3, layout, s["d"], s["sx"], s["sw"], act=act[c["act"]],
                              bias=s["bias"], residual=s["residual"], pre=s["pre"], fd=fmt, scale_d=s["scale_d"] if codes else None,
                              amax_out=s["amax"] if codes else None)
        out = [s["d"].view(view), s["amax"]] if codes else [s["d"]]
        return out + ([s["pre"]] if c["pre"] else [])
    if c["op"] == "epilogue_backward":
        api.fp8_epilogue_backward(s["dy"], s["pre"], s["dz"], act=act[c["act"]], fd=fmt, scale_d=s["scale_d"] if fmt is not None else None,
                                  dbias=s["dbias"], amax_out=s["amax"] if fmt is not None else None)
        return [s["dz"].view(view), s["dbias"], s["amax"]] if fmt is not None else [s["dz"], s["dbias"]]
    if c["op"] == "gated":
        codes = fmt is not None
        api.fp8_gemm_gated(s["x"], api.E4M3, api.MAJOR_K, s["wg"], s["wu"], api.E4M3, layout, s["h"], s["sx"], s["sg"], s["su"],
                           act=act[c["act"]], gate=s["gate"], up=s["up"], fd=fmt, scale_d=s["scale_d"] if codes else None,
                           amax_out=s["amax"] if codes else None)
        out = [s["h"].view(view), s["amax"]] if codes else [s["h"]]
        return out + ([s["gate"], s["up"]] if c["save"] else [])
    if c["op"] == "gated_backward":
        codes = fmt is not None
        # W_d is stored [d_out, d_in]: the contraction runs over its contiguous index
        api.fp8_gemm_gated_backward(s["dy"], api.E5M2, api.MAJOR_K, s["wd"], api.E4M3, api.MAJOR_K if c["weight"] == "kn" else api.MAJOR_MN,
                                    s["gate"], s["up"], s["dg"], s["du"], s["sy"], s["sd"], act=act[c["act"]], fd=fmt,
                                    scale_d=s["scale_d"] if codes else None, amax_out=s["amax"] if codes else None)
        out = [s["dg"].view(view), s["du"].view(view), s["amax"]] if codes else [s["dg"], s["du"]]
        if c["chain"]:
            api.fp8_gemm(s["dgu"], fmt, api.MAJOR_K, s["wgu"], api.E4M3, api.MAJOR_K, s["dx"], s["inv_d"], s["sgu"])
            api.fp8_gemm(s["x"], api.E4M3, api.MAJOR_MN, s["dgu"], fmt, api.MAJOR_MN, s["dw"], s["sx"], s["inv_d"])
            out += [s["dx"], s["dw"]]
        return out
    api.fp8_grad_clip(s["plan"], s["max_norm"], s["norm"])
    return [s["norm"], s["flat"]]


# ---- the plain form -------------------------------------------------------------------------------------------------

def _value(codes, fmt):
    return codes.view(F8[fmt]).float()


def _weight(s, key):
    """decoded weights as [d_in, d_out]"""
    w = _value(s[key], "e4m3")
    return w if s["case"]["weight"] == "kn" else w.t()


def _act(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return z.clamp(min=0.0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1.0 + torch.exp(-z))


def _act_grad(z, kind):
    if kind == "none":
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0.0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    e = 1.0 / (1.0 + torch.exp(-z))
    return e * (1.0 + z * (1.0 - e))


def _store(v, out, scale):
    """[the rounded result] or [the codes' values, the largest magnitude before scaling]"""
    if out in WIDE:
        return [v.to(WIDE[out])]
    return [(v * scale).clamp(-FMAX[out], FMAX[out]).to(F8[out]), v.abs().max().reshape(1)]


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s)
    if c["op"] == "epilogue":
        z = torch.mm(_value(s["x"], "e4m3"), _weight(s, "w")) * (s["sx"] * s["sw"])
        if c["bias"]:
            z = z + s["bias"].float()
        v = _act(z, c["act"])
        if c["residual"]:
            v = v + s["residual"].float()
        return _store(v, c["out"], s["scale_d"]) + ([z.to(torch.bfloat16)] if c["pre"] else [])
    if c["op"] == "epilogue_backward":
        dz = s["dy"].float() * _act_grad(s["pre"].float(), c["act"])
        out = _store(dz, c["out"], s["scale_d"])
        return out[:1] + [dz.sum(dim=0)] + out[1:]
    if c["op"] == "gated":
        x = _value(s["x"], "e4m3")
        g = torch.mm(x, _weight(s, "wg")) * (s["sx"] * s["sg"])
        u = torch.mm(x, _weight(s, "wu")) * (s["sx"] * s["su"])
        out = _store(_act(g, c["act"]) * u, c["out"], s["scale_d"])
        return out + ([g.to(torch.bfloat16), u.to(torch.bfloat16)] if c["save"] else [])
    if c["op"] == "gated_backward":
        dh = torch.mm(_value(s["dy"], "e5m2"), _weight(s, "wd").t()) * (s["sy"] * s["sd"])
        g, u = s["gate"].float(), s["up"].float()
        dg, du = dh * u * _act_grad(g, c["act"]), dh * _act(g, c["act"])
        a, b = _store(dg, c["out"], s["scale_d"]), _store(du, c["out"], s["scale_d"])
        out = [a[0], b[0]] + ([torch.maximum(a[1], b[1])] if len(a) > 1 else [])
        if c["chain"]:
            N = c["d_out"]
            full = torch.zeros(s["dgu"].shape, device=DEV)
            full[:, :N] = a[0].float()
            full[:, full.shape[1] // 2:full.shape[1] // 2 + N] = b[0].float()
            wgu = _value(s["wgu"], "e4m3")
            out.append((torch.mm(full, wgu.t()) * (s["inv_d"] * s["sgu"])).to(torch.bfloat16))
            out.append((torch.mm(_value(s["x"], "e4m3").t(), full) * (s["sx"] * s["inv_d"])).to(torch.bfloat16))
        return out
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt().reshape(1)
    coef = torch.where(norm <= s["max_norm"], torch.ones_like(norm), s["max_norm"] / norm)
    _ = [to.copy_(t.float() * coef) for t, to in zip(s["grads"], s["clipped"])]
    return [norm, s["flat"]]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _table64(fmt):
    """The 256 values of a format from its bit fields: sign, exponent, mantissa."""
    mbits, bias = (3, 7) if fmt == "e4m3" else (2, 15)
    got = []
    for c in range(256):
        e, m = (c & 0x7F) >> mbits, c & ((1 << mbits) - 1)
        v = math.ldexp(m, 1 - bias - mbits) if e == 0 else math.ldexp((1 << mbits) + m, e - bias - mbits)
        got.append(-v if c & 0x80 else v)
    return torch.tensor(got, dtype=torch.float64, device=DEV)


def _decode64(codes, fmt):
    return torch.index_select(_table64(fmt), 0, codes.reshape(-1).int()).reshape(codes.shape)


def _encode64(y, fmt):
    """Nearest value of the format, ties to the even significand, saturating."""
    mbits, emin = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(y)[1].to(torch.float64) - 1
    step = torch.exp2(e.clamp(min=float(emin)) - mbits)
    return (torch.round(y / step) * step).clamp(-FMAX[fmt], FMAX[fmt])


def _sigmoid64(t):
    return torch.reciprocal(torch.exp(-t) + 1)


def _act64(z, kind):
    """(act(z), act'(z))"""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        on = (z > 0).to(torch.float64)
        return z * on, on
    if kind == "gelu":
        cdf = torch.erfc(-z / math.sqrt(2.0)) / 2
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        # (1 + tanh t)/2 is the logistic function of 2t
        k = 2 * math.sqrt(2 / math.pi)
        p = _sigmoid64(k * (z + 0.044715 * z ** 3))
        return z * p, p + z * p * (1 - p) * k * (1 + 0.134145 * z ** 2)
    p = _sigmoid64(z)
    return z * p, p + z * p * (1 - p)


def _kept64(v, out, scale):
    return [v] if out in WIDE else [_encode64(v * scale.double(), out), v.abs().max().reshape(1)]


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "clip":
        squares = [torch.dot(t.double(), t.double()) for t in s["grads"]]
        norm = torch.sqrt(sum(squares)).reshape(1)
        coef = min(1.0, s["max_norm"] / float(norm))
        room = s["flat"].numel()
        return [norm, torch.cat([torch.nn.functional.pad(t.double() * coef, (0, -t.numel() % (8 if c["out"] == "bf16" else 4))) for t in s["grads"]])[:room]]
    if c["op"] == "epilogue_backward":
        dz = s["dy"].double() * _act64(s["pre"].double(), c["act"])[1]
        out = _kept64(dz, c["out"], s["scale_d"])
        return out[:1] + [dz.sum(0)] + out[1:]

    def weights64(key):
        w = _decode64(s[key], "e4m3")
        return w if c["weight"] == "kn" else w.T

    if c["op"] == "epilogue":
        z = (_decode64(s["x"], "e4m3") @ weights64("w")) * (s["sx"].double() * s["sw"].double())
        z = z if s["bias"] is None else z + s["bias"].double()
        v = _act64(z, c["act"])[0]
        v = v if s["residual"] is None else v + s["residual"].double()
        return _kept64(v, c["out"], s["scale_d"]) + ([z] if c["pre"] else [])
    if c["op"] == "gated":
        x = _decode64(s["x"], "e4m3")
        g = (x @ weights64("wg")) * (s["sx"].double() * s["sg"].double())
        u = (x @ weights64("wu")) * (s["sx"].double() * s["su"].double())
        return _kept64(_act64(g, c["act"])[0] * u, c["out"], s["scale_d"]) + ([g, u] if c["save"] else [])
    dh = (_decode64(s["dy"], "e5m2") @ weights64("wd").T) * (s["sy"].double() * s["sd"].double())
    a, da = _act64(s["gate"].double(), c["act"])
    dg, du = _kept64(dh * s["up"].double() * da, c["out"], s["scale_d"]), _kept64(dh * a, c["out"], s["scale_d"])
    out = [dg[0], du[0]] + ([torch.maximum(dg[1], du[1])] if len(dg) > 1 else [])
    if c["chain"]:
        pad = s["dgu"].shape[1] // 2 - c["d_out"]
        full = torch.nn.functional.pad(torch.stack([dg[0], du[0]], dim=1), (0, pad)).reshape(c["tokens"], -1)
        out.append((full @ _decode64(s["wgu"], "e4m3").T) * (s["inv_d"].double() * s["sgu"].double()))
        out.append((_decode64(s["x"], "e4m3").T @ full) * (s["sx"].double() * s["inv_d"].double()))
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    c = case
    size = {"bf16": 2, "f32": 4, "e4m3": 1, "e5m2": 1, "": 0}
    if c["op"] == "clip":
        n = sum(c["big"] if i % 2 == 0 else c["small"] for i in range(c["count"]))
        return {"bytes": n * (size[c["inp"]] + size[c["out"]]), "flops": 3 * n}
    T, N = c["tokens"], c["d_out"]
    if c["op"] == "epilogue_backward":
        return {"bytes": T * N * (2 * size[c["wide"]] + size[c["out"]]) + 4 * N, "flops": 20 * T * N}
    K = c["d_in"]
    if c["op"] == "epilogue":
        return {"bytes": T * K + K * N + T * N * (size[c["out"]] + size[c["residual"]] + (2 if c["pre"] else 0)) + (2 * N if c["bias"] else 0),
                "flops": 2 * T * N * K}
    if c["op"] == "gated":
        return {"bytes": T * K + 2 * K * N + T * N * (size[c["out"]] + (4 if c["save"] else 0)), "flops": 4 * T * N * K}
    need = {"bytes": T * K + K * N + T * N * (4 + 2 * size[c["out"]]), "flops": 2 * T * N * K}
    if c["chain"]:
        need["bytes"] += 2 * N * K + 2 * T * K + T * K + 4 * N * K
        need["flops"] += 8 * T * N * K
    return need
