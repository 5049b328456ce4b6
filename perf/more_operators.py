"""What stands around the linear operators of a transformer layer: bias, activation and residual in the product's epilogue,
and the norms of queries and keys for each head with the rotation by position.

A case is one of
  linear      Y = act(X W + b) + R, W in N shards, cut into k slices; Z = X W + b too where a backward pass follows;
  linear_bwd  its gradients: dZ = dY act'(Z), db = sum over tokens of dZ, dX = dZ W^T, dW = X^T dZ (dR is dY);
  qk          every head of the queries and keys divided by its root mean square, times a learned weight, then rotated:
              pairs of elements turn by position times the pair's frequency;
  qk_bwd      its gradients: of queries and keys, and of the two weights.

The pairs of a rotation over the first r elements of a head are (i, i + r/2), or (2 i, 2 i + 1) where the case is interleaved.
"""
from __future__ import annotations

import math
from typing import Dict, List

import torch

own = False

EPS = 1e-6
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ------------------------------------------------------------------------------------------------ cases
def _linear(op, name, T, I, O, N, k=1, act="none", bias="bf16", residual=False, z=False, split="out") -> Dict:
    return {"name": name, "op": op, "T": T, "I": I, "O": O, "N": N, "k": k, "act": act, "bias": bias, "residual": residual, "z": z,
            "split": split}


def _qk(op, name, T, heads, kv_heads, D, rotary=None, interleaved=False, base=10000.0, weight="bf16", far=8192) -> Dict:
    return {"name": name, "op": op, "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "rotary": D if rotary is None else rotary,
            "interleaved": interleaved, "base": base, "weight": weight, "far": far}


def listed() -> List[Dict]:
    return [
        # serving: one token of one sequence through the wide operator and its activation
        _linear("linear", "linear-t1-4096x16384", 1, 4096, 16384, 8, act="gelu_tanh"),
        # a batch of 33 sequences, a token each, through the narrow one onto the residual stream
        _linear("linear", "linear-t33-16384x4096", 33, 16384, 4096, 8, residual=True),
        # a prompt that no tile divides
        _linear("linear", "linear-t500-2560x10240", 500, 2560, 10240, 8, act="silu", bias="f32"),
        # training, the wide operator of a small feed-forward layer in four slices, Z kept for the backward pass
        _linear("linear", "linear-t8192-1024x4096", 8192, 1024, 4096, 8, k=4, act="gelu", z=True),
        # training, the widest operator's narrow half: a long reduction in eight slices, onto the residual stream
        _linear("linear", "linear-t4096-32768x8192", 4096, 32768, 8192, 8, k=8, residual=True),
        # the smallest backward pass
        _linear("linear_bwd", "linear_bwd-t128-256x1024", 128, 256, 1024, 2, act="relu"),
        # the backward passes of a small and of a middling layer's wide operator
        _linear("linear_bwd", "linear_bwd-t8192-1024x4096", 8192, 1024, 4096, 8, k=4, act="gelu"),
        _linear("linear_bwd", "linear_bwd-t16384-2560x10240", 16384, 2560, 10240, 8, k=4, act="gelu_tanh", bias="f32"),
        # serving: the queries and keys of one token far into a sequence; training: those of a full batch
        _qk("qk", "qk-t1-32x128", 1, 32, 8, 128, base=500000.0, far=131072),
        _qk("qk", "qk-t8192-32x128", 8192, 32, 32, 128),
        # heads of 80 elements, half of each rotated, in a batch that nothing divides; a full batch with shared key heads
        _qk("qk_bwd", "qk_bwd-t1001-32x80", 1001, 32, 32, 80, rotary=32, interleaved=True, weight="f32"),
        _qk("qk_bwd", "qk_bwd-t8192-32x128", 8192, 32, 8, 128),
    ]


def _log(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> Dict:
    op = rng.choice(["linear", "linear", "linear", "linear_bwd", "linear_bwd", "qk", "qk", "qk_bwd"])
    if op.startswith("linear"):
        most = 1.1e12 if op == "linear" else 4.2e11  # products that the largest listed cases make
        while True:
            T = rng.choice([_log(rng, 1, 64), _log(rng, 1, 4096), _log(rng, 128, 16384)])
            I, O = 8 * _log(rng, 32, 4096), 8 * _log(rng, 32, 4096)
            if T * I * O <= most and I * O <= 2 ** 28 and T * (I + O) <= 2 ** 28:
                break
        k, split = rng.choice([1, 1, 2, 4, 8]), rng.choice(["out", "out", "in"])
        cut = O if split == "out" else I
        while cut % (8 * k):
            k //= 2
        c = _linear(op, "", T, I, O, rng.choice([1, 2, 4, 8]), k=k, act=rng.choice(ACTIVATIONS), split=split,
                    bias=rng.choice(["bf16", "bf16", "f32", "none"]))
        if op == "linear":
            c.update(residual=rng.random() < 0.5, z=rng.random() < 0.5)
    else:
        while True:
            T, D = rng.choice([_log(rng, 1, 64), _log(rng, 1, 8192)]), rng.choice([32, 64, 80, 96, 128, 128, 256])
            kv = rng.choice([1, 2, 4, 8, 16, 32])
            heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
            if heads <= 64 and T * (heads + kv) * D <= (6.7e7 if op == "qk" else 4.1e7):
                break
        c = _qk(op, "", T, heads, kv, D, rotary=rng.choice([D, D, D // 32 * 16]), interleaved=rng.random() < 0.4,
                base=rng.choice([10000.0, 500000.0]), weight=rng.choice(["bf16", "bf16", "f32"]), far=_log(rng, 256, 1 << 20))
    del c["name"]
    return c


def work(case) -> Dict:
    if case["op"].startswith("linear"):
        T, I, O = case["T"], case["I"], case["O"]
        b = {"none": 0, "bf16": 2, "f32": 4}[case["bias"]] * O
        if case["op"] == "linear":
            return {"bytes": 2 * (T * I + I * O + T * O * (1 + case["residual"] + case["z"])) + b, "flops": 2 * T * I * O}
        z = 2 if case["act"] != "none" else 0  # Z read, dZ written
        return {"bytes": 2 * (2 * T * I + 2 * I * O + T * O * (1 + z)) + b, "flops": 4 * T * I * O}
    n = case["T"] * (case["heads"] + case["kv_heads"]) * case["D"]
    more = 8 * case["T"] + 4 * case["rotary"]
    w = {"bf16": 2, "f32": 4}[case["weight"]] * 2 * case["D"]
    if case["op"] == "qk":
        return {"bytes": 4 * n + more + w, "flops": 7 * n}
    return {"bytes": 6 * n + more + 2 * w, "flops": 16 * n}


# ------------------------------------------------------------------------------------------------ inputs
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(case, seed: int) -> Dict:
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)

    s = {"case": dict(case)}
    if case["op"].startswith("linear"):
        T, I, O, N = case["T"], case["I"], case["O"], case["N"]
        L = -(-I * O // N)
        flat = torch.zeros(N * L, dtype=torch.bfloat16, device="cuda")
        flat[:I * O] = normal(I * O, std=0.02)
        s["w"] = [w.clone() for w in flat.split(L)]
        s["X"] = normal(T, I)
        s["bias"] = None if case["bias"] == "none" else normal(O, std=0.1, dtype=_DTYPE[case["bias"]])
        if case["op"] == "linear":
            s["R"] = normal(T, O) if case["residual"] else None
        else:
            s["dY"] = normal(T, O)
            s["Z"] = None if case["act"] == "none" else normal(T, O, std=0.02 * math.sqrt(I))
        return s
    T, H, G, D = case["T"], case["heads"], case["kv_heads"], case["D"]
    s["qkv"] = normal(T, (H + 2 * G) * D)
    s["gq"], s["gk"] = (normal(D, std=0.2, dtype=torch.float32).add_(1.0).to(_DTYPE[case["weight"]]) for _ in range(2))
    # tokens of a few sequences one after another, each from some position on
    pieces = torch.randint(1, 9, (1,), generator=gen, device="cuda").item()
    at = torch.arange(T, device="cuda", dtype=torch.int64)
    piece = at * pieces // T
    starts = torch.randint(0, max(1, case["far"] - T), (pieces,), generator=gen, device="cuda", dtype=torch.int64)
    s["positions"] = starts[piece] + at - (piece * T + pieces - 1) // pieces
    r = case["rotary"]
    s["freqs"] = case["base"] ** (-2.0 * torch.arange(r // 2, device="cuda", dtype=torch.float64) / r)
    if case["op"] == "qk_bwd":
        s["dq_out"], s["dk_out"] = normal(T, H, D), normal(T, G, D)
    return s


def _heads(case, flat):
    """The queries and the keys in rows of queries, keys and values."""
    H, G, D = case["heads"], case["kv_heads"], case["D"]
    return flat[:, :H * D].unflatten(1, (H, D)), flat[:, H * D:(H + G) * D].unflatten(1, (G, D))


def prepare(case, seed: int):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2209_13258_amd as osdp

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s["osdp"] = osdp
    if case["op"].startswith("linear"):
        T, I, O, N, k = (case[x] for x in ("T", "I", "O", "N", "k"))
        bwd = case["op"] == "linear_bwd"
        cut = osdp.OSDP_SPLIT_OUT_FEATURES if case["split"] == "out" else osdp.OSDP_SPLIT_IN_FEATURES
        s["plan"] = osdp.Plan([k], split_dim_per_op=[cut])
        need, _ = osdp.osdp_split_linear_epilogue_workspace_bytes(T, I, O, N, k, bwd, plan=s["plan"])
        s["ws"] = empty(max(need, 256), dtype=torch.uint8)
        act = getattr(osdp, "OSDP_ACT_" + case["act"].upper())
        if bwd:
            s["dX"], s["dw"] = empty(T, I), [torch.zeros_like(w) for w in s["w"]]
            s["dZ"] = None if s["Z"] is None else empty(T, O)
            s["db"] = None if s["bias"] is None else torch.empty_like(s["bias"])
            s["epilogue"] = osdp.EpilogueGrad(activation=act, z=s["Z"], dz=s["dZ"], dbias=s["db"])
        else:
            s["Y"] = empty(T, O)
            s["Z"] = empty(T, O) if case["z"] else None
            s["epilogue"] = osdp.Epilogue(bias=s["bias"], activation=act, residual=s["R"], z=s["Z"])
        return s
    T, H, G, D = case["T"], case["heads"], case["kv_heads"], case["D"]
    s["q"], s["k"] = _heads(case, s["qkv"])
    if case["op"] == "qk":
        s["q_out"], s["k_out"] = empty(T, H, D), empty(T, G, D)
    else:  # (beside the values' gradient, as the product's backward pass takes them)
        s["dqkv"] = torch.zeros_like(s["qkv"])
        s["dq"], s["dk"] = _heads(case, s["dqkv"])
        s["dgq"], s["dgk"] = torch.empty_like(s["gq"]), torch.empty_like(s["gk"])
        s["ws"] = empty(max(osdp.osdp_qk_norm_rope_bwd_workspace_bytes(T, H, G, D), 256), dtype=torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _act(name: str, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_slope(name: str, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        p = torch.sigmoid(c * (z + 0.044715 * z * z * z))
        return p + z * p * (1 - p) * c * (1 + 3 * 0.044715 * z * z)
    p = torch.sigmoid(z)
    return p + z * p * (1 - p)


def _plain_linear(s):
    c = s["case"]
    w = torch.cat(s["w"])[:c["I"] * c["O"]].view(c["I"], c["O"]).float()
    x = s["X"].float()
    if c["op"] == "linear":
        z = x @ w
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(c["act"], z)
        if s["R"] is not None:
            y = y + s["R"].float()
        out = {"Y": y.to(torch.bfloat16)}
        if c["z"]:
            out["Z"] = z.to(torch.bfloat16)
        return out
    dz = s["dY"].float()
    if s["Z"] is not None:
        dz = dz * _act_slope(c["act"], s["Z"].float())
    flat = torch.zeros(sum(p.numel() for p in s["w"]), dtype=torch.bfloat16, device="cuda")
    flat[:c["I"] * c["O"]] = (x.t() @ dz).to(torch.bfloat16).reshape(-1)
    out = {"dX": (dz @ w.t()).to(torch.bfloat16), "dW": list(flat.split(s["w"][0].numel()))}
    if s["Z"] is not None:
        out["dZ"] = dz.to(torch.bfloat16)
    if s["bias"] is not None:
        out["db"] = dz.double().sum(0).to(s["bias"].dtype)
    return out


def _turn(case, x, cos, sin):
    """Every head's first elements turned in pairs by the angles whose cosines and sines these are."""
    r = case["rotary"]
    turned, rest = x[..., :r], x[..., r:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)
    a, b = turned[..., :r // 2], turned[..., r // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _plain_qk(s):
    c = s["case"]
    angle = (s["positions"].double()[:, None] * s["freqs"])[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {}
    for name, x, g in zip("qk", _heads(c, s["qkv"]), (s["gq"], s["gk"])):
        x, g = x.float(), g.float()
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if c["op"] == "qk":
            out[name] = _turn(c, x * rstd * g, cos, sin).to(torch.bfloat16)
        else:
            dn = _turn(c, s[f"d{name}_out"].float(), cos, -sin)
            xh = x * rstd
            out[f"dg{name}"] = (dn * xh).double().sum((0, 1)).to(s[f"g{name}"].dtype)
            t = dn * g
            out[f"d{name}"] = (rstd * (t - xh * (t * xh).mean(-1, keepdim=True))).to(torch.bfloat16)
    return out


def run(s):
    c = s["case"]
    if own:
        return _run_own(s)
    return _plain_linear(s) if c["op"].startswith("linear") else _plain_qk(s)


# ------------------------------------------------------------------------------------------------ the framework's calls
def _run_own(s):
    c, osdp = s["case"], s["osdp"]
    if c["op"] == "linear":
        osdp.osdp_split_linear_fwd_epilogue(s["X"], s["w"], s["Y"], c["k"], s["ws"], epilogue=s["epilogue"], plan=s["plan"])
        return {"Y": s["Y"], "Z": s["Z"]} if c["z"] else {"Y": s["Y"]}
    if c["op"] == "linear_bwd":
        osdp.osdp_split_linear_bwd_epilogue(s["X"], s["dY"], s["w"], s["dX"], s["dw"], c["k"], s["ws"], epilogue=s["epilogue"],
                                            plan=s["plan"])
        out = {"dX": s["dX"], "dW": s["dw"]}
        if s["Z"] is not None:
            out["dZ"] = s["dZ"]
        if s["bias"] is not None:
            out["db"] = s["db"]
        return out
    how = dict(positions=s["positions"], freqs=s["freqs"], q_weight=s["gq"], k_weight=s["gk"], eps=EPS, interleaved=c["interleaved"])
    if c["op"] == "qk":
        osdp.osdp_qk_norm_rope_fwd(s["q"], s["k"], s["q_out"], s["k_out"], **how)
        return {"q": s["q_out"], "k": s["k_out"]}
    osdp.osdp_qk_norm_rope_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["dgq"], s["dgk"], s["ws"], **how)
    return {"dgq": s["dgq"], "dq": s["dq"], "dgk": s["dgk"], "dk": s["dk"]}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed: int):
    """What the definitions say, in 64 bits."""
    s = _inputs(case, seed)
    if case["op"].startswith("linear"):
        return _exact_linear(case, s)
    D, r = case["D"], case["rotary"]
    # the rotation of a head as complex numbers times exp(i angle)
    unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double().outer(s["freqs"]))[:, None]
    first = torch.arange(0, r, 2, device="cuda") if case["interleaved"] else torch.arange(r // 2, device="cuda")
    second = first + (1 if case["interleaved"] else r // 2)

    def rotate(x, by):
        w = torch.complex(x[..., first], x[..., second]) * by
        y = x.clone()
        y[..., first], y[..., second] = w.real, w.imag
        return y

    H, G = case["heads"], case["kv_heads"]
    out = {}
    for name, x, g in (("q", s["qkv"][:, :H * D].reshape(-1, H, D), s["gq"]), ("k", s["qkv"][:, H * D:(H + G) * D].reshape(-1, G, D), s["gk"])):
        x, g = x.double(), g.double()
        size = ((x ** 2).sum(-1, keepdim=True) / D + EPS) ** 0.5
        if case["op"] == "qk":
            out[name] = rotate(x / size * g, unit)
            continue
        dn = rotate(s[f"d{name}_out"].double(), unit.conj())
        out[f"dg{name}"] = (dn * x / size).sum((0, 1))
        out[f"d{name}"] = dn * g / size - x * (dn * g * x).sum(-1, keepdim=True) / (D * size ** 3)
    return out


def _exact_linear(case, s):
    I, O = case["I"], case["O"]
    w = torch.cat(s["w"])[:I * O].reshape(I, O).double()
    x = s["X"].double()
    if case["op"] == "linear":
        z = torch.mm(x, w)
        del x, w
        if s["bias"] is not None:
            z += s["bias"].double()
        a = z
        if case["act"] == "relu":
            a = z.clamp(min=0)
        elif case["act"] == "gelu":
            a = z * 0.5 * torch.erfc(z / -math.sqrt(2))
        elif case["act"] == "gelu_tanh":
            a = z / (1 + torch.exp(-math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)))
        elif case["act"] == "silu":
            a = z / (1 + torch.exp(-z))
        out = {"Y": a if s["R"] is None else a + s["R"].double()}
        if case["z"]:
            out["Z"] = z
        return out
    dz = s["dY"].double()
    if s["Z"] is not None:
        z = s["Z"].double()
        if case["act"] == "relu":
            dz[z <= 0] = 0
        elif case["act"] == "gelu":
            dz *= 0.5 * torch.erfc(z / -math.sqrt(2)) + z * torch.exp(-z ** 2 / 2) * (2 * math.pi) ** -0.5
        else:  # z sigma(u(z)): the slope is sigma + z u' sigma (1 - sigma)
            c = math.sqrt(8 / math.pi)
            u, du = (z, 1.0) if case["act"] == "silu" else (c * (z + 0.044715 * z ** 3), c * (1 + 0.134145 * z ** 2))
            up = 1 / (1 + torch.exp(-u))
            dz *= up + z * du * up / (1 + torch.exp(u))
        del z
    out = {"dX": torch.mm(dz, w.t().contiguous())}
    del w
    flat = torch.zeros(sum(p.numel() for p in s["w"]), dtype=torch.float64, device="cuda")
    flat[:I * O] = torch.mm(x.t().contiguous(), dz).view(-1)
    out["dW"] = list(flat.split(s["w"][0].numel()))
    if s["Z"] is not None:
        out["dZ"] = dz
    if s["bias"] is not None:
        out["db"] = dz.sum(0)
    return out
