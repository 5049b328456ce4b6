"""The operators around a sharded weight: its update by AdamW, and its product in 8-bit integers.

A case is one of
  sumsq     the sum of squares of many gradients, in 64 bits: what clipping by the global norm goes by;
  adamw     one AdamW step over many tensors, the moments held in 32 or in 8 bits;
  quantize  the bf16 shards of a weight to 8-bit integers with a scale for each output channel;
  linear    Y = X . W with W in 8-bit integers, every token of X brought to 8 bits on the way.

Formats that both sides share:
  weights  q[o, i] = round(W[i, o] * 127 / amax_o), halves away from zero, stored [O x I] in N flat shards of
           ceil(I O / N); scale_o = amax_o / 127.  Tokens alike: x[t, i] = round(X[t, i] * 127 / amax_t).
  moments  in 8 bits: blocks of 128 elements share a power of two (one byte: the exponent of the block's largest binade,
           biased by 127; 0: the block is zero); m has a sign, 4 exponent and 3 fraction bits, v 5 and 3, both with
           gradual underflow; rounding is stochastic, from a counter that is hashed with the seed, the step and the
           tensor's place; a positive v stays positive.
"""
from __future__ import annotations

import math
from typing import Dict, List

import torch

own = False

BLOCK = 128
B1, B2, EPS, LR, DECAY = 0.9, 0.95, 1e-8, 1e-4, 0.1
SEED = 220913258
OPERATORS = {  # as (in-features, out-features) in units of the hidden size and the inner size
    "linear": lambda h, f: [(h, f)],
    "ffn": lambda h, f: [(h, f), (f, h)],
    "layer": lambda h, f: [(h, 3 * h), (h, h), (h, f), (f, h)],
}


# ------------------------------------------------------------------------------------------------ cases
def _tensors(op, name, layout, h, f, layers, N, vectors=0, odd=0, packed=False, **more) -> Dict:
    return {"name": name, "op": op, "layout": layout, "h": h, "f": f, "layers": layers, "N": N, "vectors": vectors, "odd": odd,
            "packed": packed, **more}


def _adamw(name, *shape, state=32, param="master", grad="bf16", clip=True, step=10, **more) -> Dict:
    return _tensors("adamw", name, *shape, state=state, param=param, grad=grad, clip=clip, step=step, **more)


def _weight(op, name, I, O, N, **more) -> Dict:
    return {"name": name, "op": op, "I": I, "O": O, "N": N, **more}


def listed() -> List[Dict]:
    return [
        # the norm of one small operator's gradient: two launches' latency
        _tensors("sumsq", "sumsq-256x1024", "linear", 256, 1024, 1, 2, grad="bf16"),
        # the norm of two layers' gradients before a step, every shard on this card
        _tensors("sumsq", "sumsq-layer-h4096-x2", "layer", 4096, 16384, 2, 8, grad="bf16"),
        # the smallest step: one operator in two shards
        _adamw("adamw32-256x1024", "linear", 256, 1024, 1, 2),
        # a layer in mixed precision: bf16 weights, fp32 master copies and moments
        _adamw("adamw32-layer-h2560", "layer", 2560, 10240, 1, 8, vectors=4),
        # the same with moments in 8 bits
        _adamw("adamw8-layer-h2560", "layer", 2560, 10240, 1, 8, vectors=4, state=8),
        # as little memory as it takes: bf16 weights without a master copy, moments in 8 bits, vectors of odd lengths
        _adamw("adamw8-bf16-layer-h4096", "layer", 4096, 16384, 1, 8, vectors=6, odd=3, state=8, param="bf16"),
        # a small feed-forward weight, and the largest one
        _weight("quantize", "quantize-1024x4096", 1024, 4096, 8),
        _weight("quantize", "quantize-8192x32768", 8192, 32768, 8),
        # serving, one token of one sequence; a batch of sequences; a prompt that no tile divides; a full batch
        _weight("linear", "linear-t1-4096x16384", 4096, 16384, 8, T=1),
        _weight("linear", "linear-t33-8192x32768", 8192, 32768, 8, T=33),
        _weight("linear", "linear-t500-2560x10240", 2560, 10240, 8, T=500),
        _weight("linear", "linear-t4096-8192x32768", 8192, 32768, 8, T=4096),
    ]


def _log(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> Dict:
    op = rng.choice(["sumsq", "adamw", "adamw", "adamw", "quantize", "linear", "linear", "linear"])
    if op in ("sumsq", "adamw"):
        layout = rng.choice(["linear", "ffn", "layer"])
        h = 8 * _log(rng, 32, 512)
        f = rng.choice([4 * h, 8 * _log(rng, 32, 2048)])
        more = {"vectors": rng.randrange(0, 8), "odd": rng.choice([0, 0, 1, 3, 5, 77]), "packed": rng.random() < 0.2}
        c = _tensors(op, "", layout, h, f, 1, rng.choice([1, 2, 3, 5, 8]), **more)
        if sum(_lengths(c)) < 1e8:
            c["layers"] = rng.choice([1, 2])
        if op == "sumsq":
            c["grad"] = rng.choice(["bf16", "bf16", "f32"])
        else:
            c.update(state=rng.choice([32, 8, 8]), param=rng.choice(["master", "master", "bf16", "f32"]),
                     grad=rng.choice(["bf16", "bf16", "f32"]), clip=rng.random() < 0.7, step=_log(rng, 1, 100000))
    else:
        N = rng.choice([1, 2, 4, 8])
        I, O = 16 * _log(rng, 16, 1024), 8 * _log(rng, 32, 2048)
        c = _weight(op, "", I, O, N)
        if op == "linear":
            c["T"] = rng.choice([_log(rng, 1, 64), _log(rng, 1, 4096), _log(rng, 1, 4096), _log(rng, 128, 4096)])
    del c["name"]
    return c


def _lengths(case) -> List[int]:
    """Elements of each tensor: the N shards of every operator (flat pieces of ceil(I O / N)), then the layer's vectors."""
    out = []
    for _ in range(case["layers"]):
        for i, o in OPERATORS[case["layout"]](case["h"], case["f"]):
            out += [-(-i * o // case["N"])] * case["N"]
        out += [case["h"] + case["odd"]] * case["vectors"]
    return out


def _starts(case) -> List[int]:
    """Where each tensor begins in the flat buffers: on multiples of 128 elements, or (packed) right behind the last."""
    at, out = 0, []
    for n in _lengths(case):
        out.append(at)
        at += n if case["packed"] else -(-n // BLOCK) * BLOCK
    return out + [at]


def work(case) -> Dict:
    if case["op"] in ("sumsq", "adamw"):
        n = sum(_lengths(case))
        g = 2 if case["grad"] == "bf16" else 4
        if case["op"] == "sumsq":
            return {"bytes": n * g + 8, "flops": 2 * n}
        p = {"master": 10, "bf16": 4, "f32": 8}[case["param"]]
        # (moments in 8 bits: both read and written, 4 / 128 bytes for their powers of two, and the values they stand for)
        s = 16 if case["state"] == 32 else 4 + 4 / BLOCK + 4
        return {"bytes": n * (g + p + s), "flops": 20 * n}
    w = case["I"] * case["O"]
    if case["op"] == "quantize":
        return {"bytes": 3 * w + 4 * case["O"], "flops": 3 * w}
    T = case["T"]
    return {"bytes": 2 * T * case["I"] + w + 4 * case["O"] + 2 * T * case["O"], "flops": 2 * T * w}


# ------------------------------------------------------------------------------------------------ inputs
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _zero_padding(case, *flat):
    starts, lengths = _starts(case), _lengths(case)
    for i, n in enumerate(lengths):
        for t in flat:
            t[starts[i] + n:starts[i + 1]] = 0


def _inputs(case, seed: int) -> Dict:
    """The numbers a case is about, alike for both sides."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(n, std):
        return torch.randn(n, generator=gen, device="cuda") * std

    s = {"case": dict(case)}
    if case["op"] in ("sumsq", "adamw"):
        total = _starts(case)[-1]
        # gradients of very different size from one 4096 elements to the next
        spread = torch.exp(1.5 * normal(-(-total // 4096), 1.0)).repeat_interleave(4096)[:total]
        grad = normal(total, 1e-3).mul_(spread)
        s["grad"] = grad.to(_DTYPE[case["grad"]])
        if case["op"] == "sumsq":
            _zero_padding(case, s["grad"])
            return s
        weight = normal(total, 0.02)
        m = normal(total, 3e-4).mul_(spread)
        v = (0.5 + torch.rand(total, generator=gen, device="cuda")).mul_(1e-6).mul_(spread).mul_(spread)
        _zero_padding(case, s["grad"], weight, m, v)
        if case["param"] == "f32":
            s["param"] = weight
        else:
            s["param"] = weight.to(torch.bfloat16)
            if case["param"] == "master":
                s["master"] = weight
        if case["state"] == 32:
            s["m"], s["v"] = m, v
        else:
            s["m8"], s["v8"], s["exps"] = (torch.empty(total, dtype=torch.uint8, device="cuda"),
                                           torch.empty(total, dtype=torch.uint8, device="cuda"), [])
            starts = _starts(case)
            for i, n in enumerate(_lengths(case)):
                a, b = starts[i], starts[i] + n
                u = torch.full((n,), 0.5, device="cuda")
                s["m8"][a:b], em = _encode(m[a:b], u, 15, 32, True)
                s["v8"][a:b], ev = _encode(v[a:b], u, 31, 48, False)
                s["m8"][b:starts[i + 1]] = 0
                s["v8"][b:starts[i + 1]] = 0
                s["exps"].append(torch.stack([em, ev], dim=1).contiguous())
        s["step"] = case["step"]
        # the norm that another pass found: about what these gradients have
        s["sumsq"] = s["grad"].double().square().sum().reshape(1) * (0.5 + torch.rand(1, generator=gen, device="cuda").double())
        s["max_norm"] = 1.0 if case["clip"] else 0.0
        return s
    I, O, N = case["I"], case["O"], case["N"]
    L = -(-I * O // N)
    scale = torch.exp(0.5 * normal(O, 1.0))
    if case["op"] == "quantize":
        w = torch.zeros(N * L, dtype=torch.bfloat16, device="cuda")
        w[:I * O] = (normal(I * O, 0.02).view(I, O) * scale).to(torch.bfloat16).view(-1)
        s["w"] = [w[j * L:(j + 1) * L].clone() for j in range(N)]
        return s
    q = torch.zeros(N * L, dtype=torch.int8, device="cuda")
    q[:I * O] = normal(I * O, 32.0).round_().clamp_(-127, 127).to(torch.int8)
    s["q"] = [q[j * L:(j + 1) * L].clone() for j in range(N)]
    s["scale"] = scale * (0.08 / 127)
    X = normal(case["T"] * I, 1.0).view(case["T"], I) * torch.exp(0.5 * normal(case["T"], 1.0)).unsqueeze(1)
    if case["T"] > 64:
        X[-case["T"] // 37:] = 0  # the padding behind a packed batch
    s["X"] = X.to(torch.bfloat16)
    return s


def prepare(case, seed: int) -> Dict:
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("sumsq", "adamw"):
        starts, lengths = _starts(case), _lengths(case)
        s["views"] = {k: [s[k][starts[i]:starts[i] + n] for i, n in enumerate(lengths)]
                      for k in ("grad", "param", "master", "m", "v", "m8", "v8") if k in s}
        if op == "sumsq":
            s["sumsq"] = torch.zeros(1, dtype=torch.float64, device="cuda")
        elif case["state"] == 8:
            total = starts[-1]
            s["m_values"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
            s["v_values"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
            for k in ("m_values", "v_values"):
                s["views"][k] = [s[k][starts[i]:starts[i] + n] for i, n in enumerate(lengths)]
    elif op == "quantize":
        s["q"] = [torch.zeros(w.numel(), dtype=torch.int8, device="cuda") for w in s["w"]]
        s["scale"] = torch.zeros(case["O"], device="cuda")
    else:
        s["Y"] = torch.zeros(case["T"], case["O"], dtype=torch.bfloat16, device="cuda")
    if own:
        import paper_2209_13258_amd as osdp
        s["osdp"] = osdp
        need = 0
        if op in ("sumsq", "adamw"):
            g = s["views"]
            if op == "sumsq":
                s["table"] = osdp.AdamWTable(grads=g["grad"])
                need = osdp.osdp_adamw_grad_sumsq_workspace_bytes(s["table"])
            else:
                s["table"] = osdp.AdamWTable(params=g["param"], grads=g["grad"], masters=g.get("master"),
                                             m=g.get("m", g.get("m8")), v=g.get("v", g.get("v8")), exps=s.get("exps"),
                                             weight_decay=DECAY)
        elif op == "quantize":
            need = osdp.osdp_split_linear_i8_quantize_workspace_bytes(case["I"], case["O"], case["N"])
        else:
            need, _ = osdp.osdp_split_linear_i8_workspace_bytes(case["T"], case["I"], case["O"], case["N"], 1)
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms
_MASK = 0xFFFFFFFF


def _mix(x):
    """32 bits stirred: of a whole number, or of a tensor of them in 64 bits."""
    x = (x * 0x9E3779B1) & _MASK
    x = x ^ (x >> 15)
    x = (x * 0x2C1B3C6D) & _MASK
    return x ^ (x >> 13)


def _random(n: int, seed: int, step: int, tensor: int):
    """Three times 16 random bits for each of a tensor's elements, as fractions of one."""
    key = _mix(_mix(_mix(_mix(seed & _MASK) ^ (seed >> 32)) ^ (step & _MASK)) ^ tensor)
    at = torch.arange(n, device="cuda", dtype=torch.int64)
    if n > 1 << 32:
        raise ValueError("the plain form counts elements in 32 bits")
    h = _mix((at + _mix(key)) & _MASK)
    p = (h * 0x297A2D39) & _MASK
    return (h & 0xFFFF).float() / 65536, (h >> 16).float() / 65536, p >> 16


def _bits(x):
    return x.view(torch.int32).to(torch.int64)


def _two(e):
    """2^e for whole e in -126 .. 127, exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _blocks(x, fill=0):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % BLOCK), value=fill).view(-1, BLOCK)


def _least(e_block, top: int, n: int):
    """The biased exponent of each element's smallest binade; any for a block of zeros."""
    least = torch.where(e_block > 0, e_block.to(torch.int64) - (top - 1), torch.full_like(e_block, 127, dtype=torch.int64))
    return least.repeat_interleave(BLOCK)[:n]


def _encode(x, u, top: int, low: int, signed: bool):
    """Codes and block exponents of fp32 values: `top` the largest exponent field, u in [0, 1) decides the rounding."""
    a = x.abs()
    most = _bits(_blocks(a).amax(dim=1))
    e_block = ((most + 0xFFFFF) >> 23).clamp(min=low)  # (the exponent that the largest one has when it is rounded up)
    e_block = torch.where(most == 0, torch.zeros_like(e_block), e_block)
    least = _least(e_block, top, x.numel())
    e = torch.maximum(_bits(a) >> 23, least)
    q = torch.floor(a * _two(130 - e) + u).to(torch.int64)
    code = (e - least) * 8 + q
    if signed:
        code = code | ((_bits(x) >> 31) & 1) << 7
    else:
        code = torch.where(a > 0, code.clamp(min=1), code)
    return code.to(torch.uint8), e_block.to(torch.uint8)


def _decode(code, e_block, top: int, signed: bool):
    c = code.to(torch.int64)
    mag = c & 127 if signed else c
    field = mag >> 3
    q = torch.where(field > 0, 8 + (mag & 7), mag)
    x = q.float() * _two(_least(e_block, top, c.numel()) + (field - 1).clamp(min=0) - 130)
    return torch.where(c > 127, -x, x) if signed else x


def _plain_adamw(s) -> Dict:
    c, g = s["case"], s["views"]
    s["step"] += 1
    t = s["step"]
    coef = torch.ones(1, device="cuda")
    if c["clip"]:
        norm = s["sumsq"].sqrt()
        coef = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    for i, grad in enumerate(g["grad"]):
        g32 = grad.float() * coef
        n = grad.numel()
        if c["state"] == 32:
            m, v = g["m"][i], g["v"][i]
        else:
            m = _decode(g["m8"][i], s["exps"][i][:, 0], 15, True)
            v = _decode(g["v8"][i], s["exps"][i][:, 1], 31, False)
        m1 = m * B1 + g32 * (1 - B1)
        v1 = v * B2 + (g32 * g32) * (1 - B2)
        source = g["master"][i] if c["param"] == "master" else g["param"][i].float()
        update = m1 / ((v1 / (1 - B2 ** t)).sqrt() + EPS) * (LR / (1 - B1 ** t))
        p1 = source * (1 - LR * DECAY) - update
        um = uv = up = None
        if c["state"] == 8 or c["param"] == "bf16":
            um, uv, up = _random(n, SEED, t, i)
        if c["param"] == "bf16":  # stochastic rounding
            g["param"][i].copy_((((_bits(p1) & _MASK) + up) >> 16 << 16).to(torch.int32).view(torch.float32).to(torch.bfloat16))
        else:
            g["param"][i].copy_(p1)
        if c["param"] == "master":
            g["master"][i].copy_(p1)
        if c["state"] == 32:
            m.copy_(m1)
            v.copy_(v1)
        else:
            m8, em = _encode(m1, um, 15, 32, True)
            v8, ev = _encode(v1, uv, 31, 48, False)
            g["m8"][i].copy_(m8)
            g["v8"][i].copy_(v8)
            s["exps"][i].copy_(torch.stack([em, ev], dim=1))
            g["m_values"][i].copy_(_decode(m8, em, 15, True))
            g["v_values"][i].copy_(_decode(v8, ev, 31, False))
    return _adamw_outputs(s)


def _adamw_outputs(s) -> Dict:
    return {k: s[k] for k in ("param", "master", "m", "v", "m_values", "v_values") if k in s}


def _round_away(x):
    return torch.sign(x) * torch.floor(x.abs() + 0.5)


def _to_8_bits(x, dim: int):
    """(whole numbers, scale) of bf16 values along `dim`; halves are found exactly in 64 bits."""
    amax = x.abs().amax(dim=dim, keepdim=True).float()
    at = torch.where(amax > 0, amax, torch.ones_like(amax)).double()
    return _round_away(x.double() * 127 / at), amax / 127


def run(s):
    c = s["case"]
    if own:
        return _run_own(s)
    if c["op"] == "sumsq":
        return torch.stack([g.double().square().sum() for g in s["views"]["grad"]]).sum()
    if c["op"] == "adamw":
        return _plain_adamw(s)
    I, O = c["I"], c["O"]
    if c["op"] == "quantize":
        q, scale = _to_8_bits(torch.cat(s["w"])[:I * O].view(I, O), 0)
        flat = torch.zeros(sum(w.numel() for w in s["w"]), dtype=torch.int8, device="cuda")
        flat[:I * O] = q.t().to(torch.int8).reshape(-1)
        return {"q": list(flat.split(s["w"][0].numel())), "scale": scale.view(-1)}
    xq, xs = _to_8_bits(s["X"], 1)
    w = torch.cat(s["q"])[:I * O].view(O, I)
    y = torch.matmul(xq.float(), w.float().t())
    return (y * xs * s["scale"]).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the framework's calls
def _run_own(s):
    c, osdp = s["case"], s["osdp"]
    if c["op"] == "sumsq":
        osdp.osdp_adamw_grad_sumsq(s["table"], s["sumsq"], s["ws"])
        return s["sumsq"][0]
    if c["op"] == "adamw":
        s["step"] += 1
        osdp.osdp_adamw_step(s["table"], lr=LR, beta1=B1, beta2=B2, eps=EPS, step=s["step"],
                             grad_sumsq=s["sumsq"] if c["clip"] else None, max_norm=s["max_norm"], seed=SEED)
        if c["state"] == 8:
            osdp.osdp_adamw_state_values(s["table"], s["views"]["m_values"], s["views"]["v_values"])
        return _adamw_outputs(s)
    if c["op"] == "quantize":
        osdp.osdp_split_linear_i8_quantize(c["I"], c["O"], s["w"], s["q"], s["scale"], s["ws"])
        return {"q": s["q"], "scale": s["scale"]}
    osdp.osdp_split_linear_i8_fwd(s["X"], s["q"], s["scale"], s["Y"], 1, s["ws"])
    return s["Y"]


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed: int):
    """What the definitions say, in 64 bits."""
    s = _inputs(case, seed)
    op = case["op"]
    if op == "sumsq":
        g = s["grad"].double()
        return torch.dot(g, g)
    if op == "quantize":
        I, O = case["I"], case["O"]
        w = torch.cat(s["w"])[:I * O].view(I, O)
        amax = w.double().abs().max(dim=0).values
        return {"q": [None] * len(s["w"]), "scale": amax / 127.0}
    if op == "linear":
        I, O = case["I"], case["O"]
        x = s["X"].double()
        amax = x.abs().max(dim=1, keepdim=True).values
        ratio = x * 127.0 / amax.clamp(min=1e-300)
        whole = torch.trunc(ratio + torch.copysign(torch.full_like(ratio, 0.5), ratio))
        w = torch.cat(s["q"])[:I * O].view(O, I).double()
        return (whole @ w.t().contiguous()) * (amax / 127.0) * s["scale"].double()
    t = case["step"] + 1
    norm = float(s["sumsq"].sqrt())
    clip = min(1.0, s["max_norm"] / norm) if case["clip"] else 1.0
    out = {}
    starts, lengths = _starts(case), _lengths(case)
    weight = s["master"] if case["param"] == "master" else s["param"]
    total = starts[-1]
    p = torch.zeros(total, dtype=torch.float64, device="cuda")
    m1, v1 = torch.zeros_like(p), torch.zeros_like(p)
    for i, n in enumerate(lengths):
        at = slice(starts[i], starts[i] + n)
        g = s["grad"][at].double() * clip
        if case["state"] == 32:
            m, v = s["m"][at].double(), s["v"][at].double()
        else:
            m = _value_64(s["m8"][at] & 127, s["exps"][i][:, 0], 15) * torch.where(s["m8"][at] > 127, -1.0, 1.0).double()
            v = _value_64(s["v8"][at], s["exps"][i][:, 1], 31)
        m1[at] = B1 * m + (1.0 - B1) * g
        v1[at] = B2 * v + (1.0 - B2) * g * g
        step = LR * (m1[at] / (1.0 - B1 ** t)) / ((v1[at] / (1.0 - B2 ** t)).sqrt() + EPS)
        p[at] = weight[at].double() * (1.0 - LR * DECAY) - step
    if case["param"] == "master":
        out["master"] = p
    out["param"] = p
    if case["state"] == 32:
        out["m"], out["v"] = m1, v1
    if case["state"] == 8 or case["param"] == "bf16":  # rounded by chance, and these are the chances
        mv, vv, pv = torch.zeros_like(p), torch.zeros_like(p), torch.zeros_like(p)
        for i, n in enumerate(lengths):
            at = slice(starts[i], starts[i] + n)
            um, uv, up = _random(n, SEED, t, i)
            if case["state"] == 8:
                mv[at] = _rounded_64(m1[at], um.double(), 15, 32)
                vv[at] = _rounded_64(v1[at], uv.double(), 31, 48)
            pv[at] = _between_64(p[at], up.double() / 65536, torch.frexp(p[at]).exponent - 8)
        if case["state"] == 8:
            out["m_values"], out["v_values"] = mv, vv
        if case["param"] == "bf16":
            out["param"] = pv
    return out


def _between_64(x, u, e):
    """x on the grid of 2^e, rounded down in size where the rest of it and u make less than one."""
    step = torch.exp2(e.double())
    return torch.copysign(torch.floor(x.abs() / step + u) * step, x)


def _rounded_64(x, u, top: int, low: int):
    size = _blocks(x.abs()).amax(dim=1)
    fraction, e = torch.frexp(size)
    e = torch.where(fraction > 0.9375, e, e - 1).clamp(min=low - 127)
    least = (e - (top - 1)).repeat_interleave(BLOCK)[:x.numel()]
    return _between_64(x, u, torch.maximum(torch.frexp(x).exponent - 1, least) - 3)


def _value_64(code, e_block, top: int):
    field, fraction = (code >> 3).double(), (code & 7).double()
    e = e_block.double().repeat_interleave(BLOCK)[:code.numel()]
    big = (8.0 + fraction) * torch.exp2(e - top + 1 + field - 1 - 130)
    small = fraction * torch.exp2(e - top + 1 - 130)
    return torch.where(e > 0, torch.where(field > 0, big, small), torch.zeros_like(big))
