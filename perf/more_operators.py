"""Cases of the end of a training step: softmax cross entropy of a vocabulary projection with its gradients, and the AdamW
step over many tensors with 32-bit or 8-bit states.

`run` computes them in their plain form (elementary torch operations in binary32 on the decoded codes, rounded once at the
end) or, where `own` is true, through the package's entry points.  FP8 results are returned as float8 views, that is as the
values the codes stand for; the scales of 8-bit states are outputs of their own.
"""
import math

import torch

own = False

DEV = "cuda"
FMAX = {"e4m3": 448.0, "e5m2": 57344.0}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
WIDE = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 256                      # elements of an 8-bit state that share a scale
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1


def listed():
    return [
        # one token scored against a large vocabulary (decoding, perplexity of a single continuation): the weights are read once
        dict(name="loss_1", op="loss", tokens=1, width=4096, vocab=131072, inp="fp8", weighted=False),
        # evaluation of a ragged batch, 16-bit projection, vocabulary of odd size
        dict(name="loss_333", op="loss", tokens=333, width=1024, vocab=50021, inp="bf16", weighted=False),
        # evaluation of a full batch of the hidden-4096 model
        dict(name="loss_4096", op="loss", tokens=4096, width=4096, vocab=65536, inp="fp8", weighted=False),
        # a whole training step of a small byte-pair model on a few tokens: launch latency counts
        dict(name="step_37", op="step", tokens=37, width=256, vocab=1000, inp="fp8", weighted=False),
        # training step of the hidden-4096 model, FP8 projection
        dict(name="step_4096", op="step", tokens=4096, width=4096, vocab=65536, inp="fp8", weighted=False),
        # the same with the projection kept in 16 bits, as many recipes do
        dict(name="step_bf16_2048", op="step", tokens=2048, width=4096, vocab=32000, inp="bf16", weighted=False),
        # backward pass alone for a short odd batch of the hidden-12288 model, tokens with weights of their own
        dict(name="grad_1001", op="grad", tokens=1001, width=12288, vocab=16001, inp="fp8", weighted=True),
        # one odd tensor
        dict(name="adamw_one", op="adamw", count=1, big=77777, small=1, param="f32", grad="f32", state="f32", copy="", step=10),
        # biases and norm weights of 48 layers: many small tensors
        dict(name="adamw_small", op="adamw", count=288, big=16384, small=4096, param="f32", grad="bf16", state="f32", copy="", step=1000),
        # feed-forward weights: 32-bit states, codes for the next step's products
        dict(name="adamw_ffn", op="adamw", count=4, big=4096 * 16384, small=4096 * 16384, param="f32", grad="bf16", state="f32", copy="e4m3", step=1000),
        # the same with 8-bit states
        dict(name="adamw_ffn_8bit", op="adamw", count=4, big=4096 * 16384, small=4096 * 16384, param="f32", grad="bf16", state="fp8", copy="e4m3", step=1000),
        # odd lengths, 16-bit parameters, 8-bit states
        dict(name="adamw_odd_8bit", op="adamw", count=37, big=1234567, small=333, param="bf16", grad="f32", state="fp8", copy="", step=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "grad", "step", "adamw", "adamw"])
    while True:
        if op == "adamw":
            c = dict(op=op, count=_log(rng, 1, 300), big=_log(rng, 64, 4096 * 16384), small=_log(rng, 1, 20000), param=rng.choice(["f32", "f32", "bf16"]),
                     grad=rng.choice(["bf16", "f32"]), state=rng.choice(["f32", "fp8"]), copy=rng.choice(["", "bf16", "e4m3", "e5m2"]), step=_log(rng, 1, 100000))
            if c["count"] * max(c["big"], c["small"]) <= 4 * 4096 * 16384:
                return c
        else:
            c = dict(op=op, tokens=_log(rng, 1, 8192), width=_log(rng, 64, 12288), vocab=_log(rng, 256, 131072), inp=rng.choice(["fp8", "fp8", "bf16"]),
                     weighted=rng.random() < 0.3)
            if c["tokens"] * c["width"] * c["vocab"] <= 4096 * 4096 * 65536 and c["width"] * c["vocab"] <= 4096 * 131072:
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


def _operand(values, inp):
    """A matrix as E4M3 codes with its inverse scale, or in bf16 with none."""
    if inp == "bf16":
        return _put(values, torch.bfloat16), None
    scale = FMAX["e4m3"] / values.abs().max().clamp(min=1e-30).reshape(1)
    return _put((values * scale).clamp(-448.0, 448.0).to(F8["e4m3"]).view(torch.uint8), torch.uint8), 1.0 / scale


def _sizes(c):
    return [c["big"] if i % 2 == 0 else c["small"] for i in range(c["count"])]


def _state_codes(values):
    """8-bit codes of a flat state and its scales, one per block."""
    top = values.view(-1, BLOCK).abs().amax(dim=1, keepdim=True)
    y = (values.view(-1, BLOCK) * (448.0 / top.clamp(min=1e-30))).clamp(-448.0, 448.0)
    return y.to(F8["e4m3"]).view(torch.uint8).reshape(-1), (top / 448.0).reshape(-1)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c, s = case, dict(case=case)
    if c["op"] != "adamw":
        T, K, V = c["tokens"], c["width"], c["vocab"]
        std = 1.2 / math.sqrt(K)
        w = torch.randn(V, K, generator=g, device=DEV) * std
        t = torch.randint(0, V, (T,), generator=g, device=DEV)
        x = torch.randn(T, K, generator=g, device=DEV)
        far = torch.rand(T, K, generator=g, device=DEV) < 0.0005
        x = torch.where(far, x.sign() * (20 + 40 * torch.rand(T, K, generator=g, device=DEV)), x)
        # a trained model favours its targets: their logits are up to 14 above the rest
        x = x + w[t] * (14 * torch.rand(T, 1, generator=g, device=DEV) / (std * std * K))
        s["x"], s["sx"] = _operand(x, c["inp"])
        s["w"], s["sw"] = _operand(w, c["inp"])
        # prompt and padding tokens do not count
        counted = torch.rand(T, generator=g, device=DEV) >= (0.05 if T > 1 else 0.0)
        s["target"] = torch.where(counted, t, torch.full_like(t, -100))
        weight = 0.25 + 1.5 * torch.rand(T, generator=g, device=DEV) if c["weighted"] else torch.ones(T, device=DEV)
        s["dloss"] = weight / T
        s["loss"], s["lse"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        if c["op"] != "loss":
            s["dx"], s["dw"] = _rows(T, K, torch.bfloat16), _rows(V, K, torch.bfloat16)
        if c["op"] == "grad":
            z = torch.mm(_value(s, "x"), _value(s, "w").t()) * _unscale(s)
            s["lse"] = torch.logsumexp(z, dim=1)
        return s
    n = _sizes(c)
    room = [-(-k // BLOCK) * BLOCK for k in n]
    total, at = sum(room), [0]
    for r in room:
        at.append(at[-1] + r)
    # every tensor is a stretch of flat buffers, as a sharded optimiser keeps them; what lies between them is zero
    ids = torch.repeat_interleave(torch.arange(len(n), device=DEV), torch.tensor([r // BLOCK for r in room], device=DEV))
    used = torch.arange(total, dtype=torch.int32, device=DEV).view(-1, BLOCK) - torch.tensor(at[:-1], dtype=torch.int32, device=DEV)[ids].unsqueeze(1)
    used = (used < torch.tensor(n, dtype=torch.int32, device=DEV)[ids].unsqueeze(1)).view(-1)

    def flat(values):
        return torch.where(used, values, torch.zeros_like(values))

    s["ids"] = ids
    s["decay"] = torch.tensor([DECAY if i % 2 == 0 else 0.0 for i in range(len(n))], device=DEV)
    s["p"] = flat(torch.randn(total, generator=g, device=DEV) * 0.02).to(WIDE[c["param"]])
    m = torch.randn(total, generator=g, device=DEV)
    grad = m * 1.7e-4 / (torch.randn(total, generator=g, device=DEV).square() + 0.1).sqrt()
    s["g"] = flat(grad).to(WIDE[c["grad"]])
    m = flat(0.3 * m + torch.randn(total, generator=g, device=DEV) * 0.2) * 1e-4
    r = flat(1e-5 + 1e-4 * torch.randn(total, generator=g, device=DEV).abs())
    if c["state"] == "fp8":
        (s["m"], s["ms"]), (s["v"], s["vs"]) = _state_codes(m), _state_codes(r)
    else:
        s["m"], s["v"] = m, r.square()
    s["norm"], s["max_norm"], s["seed"] = _scalar(1.7), 1.0, int(seed) * 7919 + 13
    if c["copy"]:
        s["copy"] = torch.zeros(total, dtype=WIDE.get(c["copy"], torch.uint8), device=DEV)
        s["scale"], s["amax"] = torch.full((len(n),), FMAX.get(c["copy"], 1.0) / 0.15, device=DEV), torch.zeros(len(n), device=DEV)
    if own:
        from paper_2209_05433_b200 import api

        def cut(t, per=1):
            return [t[a // per:(a + (k if per == 1 else -(-k // BLOCK) * BLOCK)) // per] for a, k in zip(at, n)]

        more = dict(exp_avg_scales=cut(s["ms"], BLOCK), exp_avg_sq_scales=cut(s["vs"], BLOCK)) if c["state"] == "fp8" else {}
        if c["copy"]:
            more.update(copies=cut(s["copy"]))
        if c["copy"] in F8:
            more.update(fmt=api.E4M3 if c["copy"] == "e4m3" else api.E5M2, scales=list(s["scale"].split(1)), amax_outs=list(s["amax"].split(1)))
        s["plan"] = api.AdamWPlan(cut(s["p"]), cut(s["g"]), cut(s["m"]), cut(s["v"]), weight_decay=[DECAY if i % 2 == 0 else 0.0 for i in range(len(n))], **more)
    return s


# ---- the package's operators ----------------------------------------------------------------------------------------

def _own(s):
    from paper_2209_05433_b200 import api
    c = s["case"]
    if c["op"] == "adamw":
        api.fp8_adamw_step(s["plan"], LR, c["step"], beta1=BETA1, beta2=BETA2, eps=EPS, seed=s["seed"], norm=s["norm"], max_norm=s["max_norm"])
        return _kept(s)
    f = api.E4M3 if c["inp"] == "fp8" else None
    if c["op"] != "grad":
        api.fp8_cross_entropy(s["x"], f, s["w"], f, s["target"], s["loss"], s["lse"], scale_inv_x=s["sx"], scale_inv_w=s["sw"])
    if c["op"] == "loss":
        return [s["loss"], s["lse"]]
    api.fp8_cross_entropy_backward(s["x"], f, s["w"], f, s["target"], s["lse"], s["dloss"], s["dx"], s["dw"], scale_inv_x=s["sx"], scale_inv_w=s["sw"])
    return ([s["loss"], s["lse"]] if c["op"] == "step" else []) + [s["dx"], s["dw"]]


def _kept(s):
    """The updated tensors of an AdamW state."""
    c = s["case"]
    out = [s["p"]] + ([s["m"].view(F8["e4m3"]), s["v"].view(F8["e4m3"]), s["ms"], s["vs"]] if c["state"] == "fp8" else [s["m"], s["v"]])
    if c["copy"] in F8:
        return out + [s["copy"].view(F8[c["copy"]]), s["amax"]]
    return out + ([s["copy"]] if c["copy"] else [])


# ---- the plain form -------------------------------------------------------------------------------------------------

def _value(s, key):
    return s[key].view(F8["e4m3"]).float() if s["case"]["inp"] == "fp8" else s[key].float()


def _unscale(s):
    return s["sx"] * s["sw"] if s["case"]["inp"] == "fp8" else 1.0


def _mix(x):
    """32-bit words to 32-bit words, by multiplications and shifted exclusive ors."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _chance(s):
    """The random numbers of an 8-bit step, in [0, 1): 16 bits for each element, from the seed, the step and its place."""
    seed, step = s["seed"] & 0xFFFFFFFFFFFFFFFF, s["case"]["step"]
    key = _mix((seed & 0xFFFFFFFF) ^ _mix((seed >> 32) ^ _mix(step & 0xFFFFFFFF)))
    word = _mix(((torch.arange(s["p"].numel() // 2, device=DEV) * 0x9E3779B1) + key) & 0xFFFFFFFF)
    return (torch.stack([word & 0xFFFF, word >> 16], dim=1).float() * (1.0 / 65536.0)).view(-1, BLOCK)


def _loss(s):
    c = s["case"]
    T, V, t = c["tokens"], c["vocab"], s["target"]
    x, w = _value(s, "x"), _value(s, "w")
    z = torch.mm(x, w.t()) * _unscale(s)
    counted = (t >= 0) & (t < V)
    at = torch.where(counted, t, torch.zeros_like(t)).unsqueeze(1)
    out, lse = [], s["lse"]
    if c["op"] != "grad":
        top = z.max(dim=1, keepdim=True)[0]
        lse = (top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True))).squeeze(1)
        out = [torch.where(counted, lse - z.gather(1, at).squeeze(1), torch.zeros_like(lse)), lse]
    if c["op"] == "loss":
        return out
    dz = torch.exp(z - lse.unsqueeze(1)).scatter_add_(1, at, torch.full((T, 1), -1.0, device=DEV))
    g = torch.where(counted, s["dloss"], torch.zeros_like(s["dloss"]))
    dz = dz * g.unsqueeze(1)
    if c["inp"] == "bf16":
        dz = dz.to(torch.bfloat16).float()
        return out + [torch.mm(dz, w).to(torch.bfloat16), torch.mm(dz.t(), x).to(torch.bfloat16)]
    # the gradient of the logits is an E5M2 tensor, scaled by the largest magnitude it can have
    scale = FMAX["e5m2"] / g.abs().max()
    dz = (dz * scale).clamp(-FMAX["e5m2"], FMAX["e5m2"]).to(F8["e5m2"]).float()
    return out + [(torch.mm(dz, w) * (s["sw"] / scale)).to(torch.bfloat16), (torch.mm(dz.t(), x) * (s["sx"] / scale)).to(torch.bfloat16)]


def _adamw(s):
    c = s["case"]
    b1, b2 = 1.0 - BETA1 ** c["step"], 1.0 - BETA2 ** c["step"]
    coef = torch.where(s["norm"] <= s["max_norm"], torch.ones_like(s["norm"]), s["max_norm"] / s["norm"])
    g, p = s["g"].float().view(-1, BLOCK) * coef, s["p"].float().view(-1, BLOCK)
    if c["state"] == "fp8":
        m = s["m"].view(F8["e4m3"]).float().view(-1, BLOCK) * s["ms"].unsqueeze(1)
        v = (s["v"].view(F8["e4m3"]).float().view(-1, BLOCK) * s["vs"].unsqueeze(1)).square()
    else:
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    r = torch.sqrt(v)
    keep = (1.0 - LR * s["decay"])[s["ids"]].unsqueeze(1)
    p = p * keep - (LR / b1) * m / (r * (1.0 / math.sqrt(b2)) + EPS)
    if c["state"] == "fp8":
        top = m.abs().amax(dim=1, keepdim=True)
        y = (m * torch.where(top > 0, 448.0 / top, torch.zeros_like(top))).clamp(-448.0, 448.0)
        s["m"].view(F8["e4m3"]).view(-1, BLOCK).copy_(y.to(F8["e4m3"]))
        s["ms"].copy_((top / 448.0).squeeze(1))
        # the root of the second moment, rounded up or down with the chance of its distance; what is not zero stays above zero
        top = r.amax(dim=1, keepdim=True)
        y = (r * torch.where(top > 0, 448.0 / top, torch.zeros_like(top))).clamp(max=448.0)
        grid = torch.exp2((torch.frexp(y)[1] - 1).clamp(min=-6).float() - 3.0)
        q = torch.floor(y / grid + _chance(s)) * grid
        q = torch.where(r > 0, q.clamp(min=2.0 ** -9), torch.zeros_like(q))
        s["v"].view(F8["e4m3"]).view(-1, BLOCK).copy_(q.to(F8["e4m3"]))
        s["vs"].copy_((top / 448.0).squeeze(1))
    else:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
    s["p"].copy_(p.view(-1))
    if c["copy"] in F8:
        q = s["p"].float().view(-1, BLOCK)
        y = (q * s["scale"][s["ids"]].unsqueeze(1)).clamp(-FMAX[c["copy"]], FMAX[c["copy"]])
        s["copy"].view(F8[c["copy"]]).copy_(y.to(F8[c["copy"]]).view(-1))
        s["amax"].zero_().scatter_reduce_(0, s["ids"], q.abs().amax(dim=1), "amax")
    elif c["copy"]:
        s["copy"].copy_(s["p"])
    return _kept(s)


def run(state):
    if own:
        return _own(state)
    return _adamw(state) if state["case"]["op"] == "adamw" else _loss(state)


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


def _grid64(y, fmt):
    """Distance of neighbouring values of the format at y."""
    mbits, emin = (3, -6) if fmt == "e4m3" else (2, -14)
    return torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp(min=emin) - mbits)


def _encode64(y, fmt):
    """Nearest value of the format, ties to the even significand, saturating."""
    step = _grid64(y, fmt)
    return (torch.round(y / step) * step).clamp(-FMAX[fmt], FMAX[fmt])


def _exact_loss(s):
    c, t = s["case"], s["target"]
    fp8 = c["inp"] == "fp8"
    x = _decode64(s["x"], "e4m3") * s["sx"].double() if fp8 else s["x"].double()
    w = _decode64(s["w"], "e4m3") * s["sw"].double() if fp8 else s["w"].double()
    z = x @ w.T
    lse = s["lse"].double() if c["op"] == "grad" else torch.logsumexp(z, 1)
    rows = torch.nonzero((t >= 0) & (t < c["vocab"])).squeeze(1)
    loss = torch.zeros_like(lse)
    loss[rows] = lse[rows] - z[rows, t[rows]]
    out = [] if c["op"] == "grad" else [loss, lse]
    if c["op"] == "loss":
        return out
    z.sub_(lse[:, None]).exp_()
    z[rows, t[rows]] -= 1.0
    g = torch.zeros_like(lse)
    g[rows] = s["dloss"].double()[rows]
    z *= g[:, None]
    if fp8:
        scale = FMAX["e5m2"] / g.abs().max()
        z = _encode64(z * scale, "e5m2") / scale
    else:
        z = z.to(torch.bfloat16).double()
    return out + [z @ w, z.T @ x]


def _exact_adamw(s):
    c = s["case"]
    ids = s["ids"]
    g = s["g"].double().view(-1, BLOCK) * min(1.0, s["max_norm"] / float(s["norm"]))
    if c["state"] == "fp8":
        m = _decode64(s["m"], "e4m3").view(-1, BLOCK) * s["ms"].double()[:, None]
        v = (_decode64(s["v"], "e4m3").view(-1, BLOCK) * s["vs"].double()[:, None]) ** 2
    else:
        m, v = s["m"].double().view(-1, BLOCK), s["v"].double().view(-1, BLOCK)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    r = v.sqrt()
    p = s["p"].double().view(-1, BLOCK)
    p = p - LR * (s["decay"].double()[ids][:, None] * p + m / (1 - BETA1 ** c["step"]) / (r / math.sqrt(1 - BETA2 ** c["step"]) + EPS))
    out = [p.view(-1)]
    if c["state"] == "fp8":
        ms, vs = m.abs().amax(1) / 448, r.amax(1) / 448
        qm = _encode64(m / ms.clamp(min=1e-300)[:, None], "e4m3")
        y = r / vs.clamp(min=1e-300)[:, None]
        step = _grid64(y, "e4m3")
        qv = (torch.floor(y / step + _chance(s).double()) * step).clamp(max=448.0)
        qv = torch.maximum(qv, (r > 0).double() / 512)
        out += [qm.view(-1), qv.view(-1), ms, vs]
    else:
        out += [m.view(-1), v.view(-1)]
    p = p.to(WIDE[c["param"]]).double() if c["param"] == "bf16" else p
    if c["copy"] in F8:
        ends = torch.cat([torch.bincount(ids).cumsum(0)])
        tops = p.abs().amax(1)
        parts = torch.tensor_split(tops, ends[:-1].cpu())
        out += [_encode64(p * s["scale"].double()[ids][:, None], c["copy"]).view(-1), torch.stack([q.max() for q in parts])]
    elif c["copy"]:
        out += [p.view(-1)]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(s) if case["op"] == "adamw" else _exact_loss(s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    c = case
    size = {"bf16": 2, "f32": 4, "fp8": 1, "e4m3": 1, "e5m2": 1, "": 0}
    if c["op"] == "adamw":
        n = sum(_sizes(c))
        state = 4 * size[c["state"]] + (16 / BLOCK if c["state"] == "fp8" else 0)
        return {"bytes": int(n * (size[c["grad"]] + 2 * size[c["param"]] + state + size[c["copy"]])), "flops": 16 * n}
    T, K, V = c["tokens"], c["width"], c["vocab"]
    need = (T + V) * K * size[c["inp"]] + 12 * T
    if c["op"] == "loss":
        return {"bytes": need + 4 * T, "flops": 2 * T * K * V}
    # the logits are not kept: the backward pass multiplies three times, a step four times, of which one could be saved by keeping them
    return {"bytes": need + 2 * (T + V) * K + 8 * T, "flops": 6 * T * K * V}
