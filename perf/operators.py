"""Cases of the operators of large language models that the framework offers: products with 4-bit weights and group scales
(linear_q4), with activations in 32, 16 or 8 bits, and the root-mean-square norm with the residual's addition (rms_norm, rms_norm_q8).

own               False: run() computes the operators in elementary torch operations; True: by the framework's calls
listed()          the named cases
draw(rng)         one more case of the same ranges
prepare(case, s)  what a program holds before the call
run(state)        one pass
work(case)        bytes and operations a pass cannot do without
exact(case, s)    what run returns, from the definition in 64 bits

Kinds of case:
  linear   y = act(x W^T + b), W held in 4 bits: codes 0..15, a scale (16 bits) and, with `zeros`, a zero point per row and group of inputs;
           x in fp32, fp16 or bf16, or in int8 with a scale per row ("row") or per row and group ("group")
  norm     h = x + r, y = h / sqrt(mean(h^2) + eps) * w, returned with h; with `q8` y in int8 with a scale per row or group
  chain    norm with an int8 output, then the linear layer that reads it
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
EPS = 1e-5


def _linear(name, m, c, k, x, y, group=128, zeros=False, scale="bf16", act="none", bias=False, xs="row"):
    return dict(name=name, kind="linear", m=m, c=c, k=k, x=x, y=y, group=group, zeros=zeros, scale=scale, act=act, bias=bias, xs=xs)


def _norm(name, m, d, x, q8="none", residual=True):
    return dict(name=name, kind="norm", m=m, c=d, x=x, q8=q8, residual=residual)


def listed():
    return [
        # the smallest call: the last classifier layer of a 16-layer image network, one image; launch and latency are all there is
        _linear("linear_m1_c4096_k1000_f32", 1, 4096, 1000, "f32", "f32", bias=True),
        # one token through a square projection
        _linear("linear_m1_c4096_k4096_bf16", 1, 4096, 4096, "bf16", "bf16"),
        # the first classifier layer of the image network, one image: the codes' way from memory
        _linear("linear_m1_c25088_k4096_f32", 1, 25088, 4096, "f32", "f32", bias=True, act="relu"),
        # the same at the batch that the framework's own benchmark runs
        _linear("linear_m32_c25088_k4096_f32", 32, 25088, 4096, "f32", "f32", bias=True, act="relu"),
        # sizes that fit no tile, with zero points and the smallest groups: a few requests decoded together
        _linear("linear_m13_c1111_k2077_f16", 13, 1111, 2077, "f16", "f16", group=32, zeros=True, scale="f16", bias=True, act="leaky"),
        # a short prompt
        _linear("linear_m300_c4096_k4096_bf16", 300, 4096, 4096, "bf16", "bf16", group=64, zeros=True),
        # the largest: a long prompt through a wide projection
        _linear("linear_m4096_c4096_k12288_bf16", 4096, 4096, 12288, "bf16", "bf16"),
        # a prompt in 8 bits, a scale for each group of inputs
        _linear("linear_m2048_c4096_k8192_i8", 2048, 4096, 8192, "i8", "bf16", zeros=True, xs="group"),
        # the norm between two layers, one token
        _norm("norm_m1_d4096_bf16", 1, 4096, "bf16"),
        # the same over a long prompt: the tensors' way from and to memory
        _norm("norm_m16384_d4096_bf16", 16384, 4096, "bf16"),
        # one token in 8 bits: the norm's 8-bit output and the projection that reads it
        dict(_linear("chain_m1_c4096_k4096_bf16", 1, 4096, 4096, "bf16", "bf16"), kind="chain"),
        # 64 requests decoded together, the same
        dict(_linear("chain_m64_c4096_k4096_bf16", 64, 4096, 4096, "bf16", "bf16"), kind="chain"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "norm", "chain"])
    if kind == "norm":
        m, d = _spread(rng, 1, 16384), _spread(rng, 64, 16384)
        m = max(1, min(m, 16384 * 4096 // d))
        return dict(kind="norm", m=m, c=d, x=rng.choice(["f32", "f16", "bf16"]), q8=rng.choice(["none", "none", "row", "group"]),
                    residual=rng.random() < 0.75)
    m, c, k = _spread(rng, 1, 4096), _spread(rng, 256, 25088), _spread(rng, 256, 16384)
    if rng.random() < 0.6:                       # most layers have round widths
        c, k = (c + 63) // 64 * 64, (k + 63) // 64 * 64
    m = max(1, min(m, 4096 * 4096 * 12288 // (c * k)))
    types = ["f32", "f16", "bf16", "bf16"] + (["i8", "i8"] if kind == "linear" else [])
    x = rng.choice(types)
    y = rng.choice(["f32", "bf16"]) if x == "i8" else x
    case = _linear("", m, c, k, x, y, group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.5, scale=rng.choice(["f16", "bf16"]),
                   act=rng.choice(["none", "none", "relu", "leaky"]), bias=rng.random() < 0.5, xs=rng.choice(["row", "group"]))
    case["kind"] = kind
    if kind == "chain" and case["y"] == "f32":   # (an 8-bit step is far above what 32 bits resolve)
        case["x"] = case["y"] = "bf16"
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 17)
    t = {}
    m, c = case["m"], case["c"]
    if case["kind"] != "linear":
        dt = TYPES[case["x"]]
        channel = 1.0 + 3.0 * (torch.rand(c, generator=gen, device="cuda") < 0.01).float()   # a few channels run larger
        t["x"] = (_normal(gen, m, c) * 0.5).to(dt)
        if case.get("residual", True):
            t["r"] = (_normal(gen, m, c) * channel).to(dt)
        t["w"] = (1.0 + 0.2 * _normal(gen, c)).to(dt)
        if case["kind"] == "norm":
            return t
    k, g = case["k"], case["group"]
    ng = (c + g - 1) // g
    # weights as a quantiser leaves them: normal values, each group's range spread over the codes
    w = _normal(gen, k, c) * (1.0 / math.sqrt(c))
    wp = torch.zeros(k, ng * g, device="cuda")
    wp[:, :c] = w
    wp = wp.view(k, ng, g)
    if case["zeros"]:
        lo, hi = wp.amin(2).clamp(max=0), wp.amax(2).clamp(min=0)
        s = ((hi - lo) / 15).to(TYPES[case["scale"]])
        z = torch.round(-lo / s.float()).clamp(0, 15)
        t["zeros"] = z.to(torch.uint8)
    else:
        s = (wp.abs().amax(2) / 7).to(TYPES[case["scale"]])
        z = torch.full((k, ng), 8.0, device="cuda")
    q = (torch.round(wp / s.float().unsqueeze(2)) + z.unsqueeze(2)).clamp(0, 15).to(torch.uint8).view(k, ng * g)[:, :c]
    if c % 2:
        q = torch.cat([q, torch.zeros(k, 1, dtype=torch.uint8, device="cuda")], 1)
    t["codes"] = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
    t["scales"] = s.contiguous()
    if case["bias"]:
        t["bias"] = 0.1 * _normal(gen, k)
    if case["kind"] == "linear":
        a = _normal(gen, m, c)
        if case["act"] == "relu":                # layers with a ReLU are fed by layers with one
            a = a.clamp(min=0)
        if case["x"] == "i8":
            cols = ng if case["xs"] == "group" else 1
            t["x_scale"] = (0.02 + 0.02 * torch.rand(m, cols, generator=gen, device="cuda"))
            if cols == 1:
                t["x_scale"] = t["x_scale"].view(m)
            t["x"] = torch.round(a * 32).clamp(-127, 127).to(torch.int8)
        else:
            t["x"] = a.to(TYPES[case["x"]])
    return t


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    if own and case["kind"] != "norm":
        from paper_2212_08815_amd import fscnn
        state["q4"] = fscnn.q4_import(state["codes"], state["scales"], state.get("zeros"), group=case["group"], c=case["c"])
    return state


# ---------------------------------------------------------------- the plain form

def _plain_weights(state):
    case = state["case"]
    c, g = case["c"], case["group"]
    codes = state["codes"]
    q = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1)[:, :c].float()
    s = state["scales"].float().repeat_interleave(g, 1)[:, :c]
    z = state["zeros"].float().repeat_interleave(g, 1)[:, :c] if "zeros" in state else 8.0
    return (q - z) * s


def _plain_linear(state, x, x_scale):
    case = state["case"]
    w = _plain_weights(state)
    xf = x.float()
    if x_scale is not None:
        xf = xf * (x_scale.view(-1, 1) if x_scale.dim() == 1 else x_scale.repeat_interleave(case["group"], 1)[:, :case["c"]])
    y = xf @ w.t()
    if "bias" in state:
        y = y + state["bias"]
    if case["act"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    elif case["act"] == "leaky":
        y = torch.where(y > 0, y, 0.1 * y)
    return y.to(TYPES[case["y"]])


def _plain_norm(state):
    h = state["x"].float()
    if "r" in state:
        h = h + state["r"].float()
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * state["w"].float()


def _plain_q8(y, group):
    m, c = y.shape
    if group:
        ng = (c + group - 1) // group
        a = torch.zeros(m, ng * group, device=y.device)
        a[:, :c] = y.abs()
        s = a.view(m, ng, group).amax(2) / 127
        wide = s.repeat_interleave(group, 1)[:, :c]
    else:
        s = y.abs().amax(1) / 127
        wide = s.view(m, 1).expand(m, c)
    q = torch.where(wide > 0, torch.round(y / wide), torch.zeros_like(y)).clamp(-127, 127).to(torch.int8)
    return q, s


def _stands_for(q, s, group):
    """The values that int8 codes with scales stand for."""
    return q * (s.view(-1, 1) if s.dim() == 1 else s.repeat_interleave(group, 1)[:, :q.shape[1]])


def _plain(state):
    case = state["case"]
    if case["kind"] == "linear":
        return _plain_linear(state, state["x"], state.get("x_scale"))
    h, y = _plain_norm(state)
    hr = (h.to(state["x"].dtype),) if "r" in state else ()
    if case["kind"] == "norm":
        if case["q8"] == "none":
            return (y.to(state["x"].dtype),) + hr
        group = 128 if case["q8"] == "group" else 0
        q, s = _plain_q8(y, group)
        return (_stands_for(q, s, group), s) + hr
    q, s = _plain_q8(y, case["group"] if case["xs"] == "group" else 0)
    return (_plain_linear(state, q, s),) + hr


def _own(state):
    from paper_2212_08815_amd import fscnn
    case = state["case"]
    if case["kind"] != "norm":
        act = dict(relu=case["act"] == "relu", leaky=0.1 if case["act"] == "leaky" else None, bias=state.get("bias"),
                   out_dtype=TYPES[case["y"]])
    if case["kind"] == "linear":
        return fscnn.linear_q4(state["q4"], state["x"], x_scale=state.get("x_scale"), **act)
    if case["kind"] == "norm" and case["q8"] == "none":
        out = fscnn.rms_norm(state["x"], state["w"], EPS, residual=state.get("r"))
        return out if "r" in state else (out,)
    group = (128 if case["q8"] == "group" else 0) if case["kind"] == "norm" else (case["group"] if case["xs"] == "group" else 0)
    out = fscnn.rms_norm_q8(state["x"], state["w"], EPS, residual=state.get("r"), group=group)
    if case["kind"] == "norm":
        return (_stands_for(out[0], out[1], group),) + tuple(out[1:])
    return (fscnn.linear_q4(state["q4"], out[0], x_scale=out[1], **act),) + tuple(out[2:])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- work and exact results

def work(case):
    m, c = case["m"], case["c"]
    byt = flops = 0
    if case["kind"] != "linear":
        e = BYTES[case["x"]]
        byt += m * c * e * (3 if case.get("residual", True) else 1) + c * e
        flops += 6 * m * c
        if case["kind"] == "norm":
            byt += m * c * (e if case["q8"] == "none" else 1)
            if case["q8"] != "none":
                byt += 4 * m * ((c + 127) // 128 if case["q8"] == "group" else 1)
            return dict(bytes=byt, flops=flops)
    k, ng = case["k"], (c + case["group"] - 1) // case["group"]
    byt += k * ((c + 1) // 2) + 2 * k * ng + (k * ng if case["zeros"] else 0) + (4 * k if case["bias"] else 0) + m * k * BYTES[case["y"]]
    if case["kind"] == "linear":
        byt += m * c * BYTES[case["x"]]
        if case["x"] == "i8":
            byt += 4 * m * (ng if case["xs"] == "group" else 1)
    return dict(bytes=byt, flops=flops + 2 * m * c * k)


def exact(case, seed):
    """From the definition, in 64 bits: rows of weights one block after the other, group by group where scales differ."""
    t = _inputs(case, seed)
    m, c = case["m"], case["c"]
    more = []
    if case["kind"] == "linear":
        x, xs = t["x"].double(), t.get("x_scale")
        xs = None if xs is None else xs.double()
    else:
        x = t["x"].double()
        if "r" in t:
            x += t["r"].double()
            more = [x.clone()]
        power = torch.linalg.vector_norm(x, dim=1) ** 2 / c
        x = x * torch.rsqrt(power + EPS)[:, None] * t["w"].double()[None]
        how = case["q8"] if case["kind"] == "norm" else case["xs"]
        if how == "none":
            return tuple([x] + more)
        step = c if how == "row" else 128 if case["kind"] == "norm" else case["group"]
        parts, scales = [], []
        for lo in range(0, c, step):
            p = x[:, lo:lo + step]
            s = p.abs().max(1).values / 127.0
            parts.append(torch.where(s[:, None] > 0, torch.round(p / s[:, None].clamp(min=1e-300)), torch.zeros_like(p)))
            scales.append(s)
        if case["kind"] == "norm":
            values = torch.cat([p * s[:, None] for p, s in zip(parts, scales)], 1)
            return tuple([values, scales[0] if how == "row" else torch.stack(scales, 1)] + more)
        x, xs = torch.cat(parts, 1), scales[0] if how == "row" else torch.stack(scales, 1)
    k, g = case["k"], case["group"]
    if xs is not None:
        for i, lo in enumerate(range(0, c, g)):
            x[:, lo:lo + g] *= xs[:, None] if xs.dim() == 1 else xs[:, i:i + 1]
    y = torch.empty(m, k, dtype=torch.float64, device="cuda")
    for lo in range(0, k, 2048):
        b = t["codes"][lo:lo + 2048]
        w = torch.empty(b.shape[0], 2 * b.shape[1], dtype=torch.float64, device="cuda")
        w[:, 0::2] = (b % 16).double()
        w[:, 1::2] = (b // 16).double()
        for i, at in enumerate(range(0, c, g)):
            w[:, at:at + g] -= t["zeros"][lo:lo + 2048, i:i + 1].double() if "zeros" in t else 8.0
            w[:, at:at + g] *= t["scales"][lo:lo + 2048, i:i + 1].double()
        y[:, lo:lo + 2048] = x @ w[:, :c].t()
    if "bias" in t:
        y += t["bias"].double()
    if case["act"] != "none":
        y = torch.where(y > 0, y, y * (0.0 if case["act"] == "relu" else 0.1))
    return y if case["kind"] == "linear" else tuple([y] + more)
