"""AdamW over many tensors, moments in 32 and 8 bits, and gradient norms, against plain implementations.

What is expected is computed on the CPU: m and v in numpy's fp32, operation by operation as the formulas have them (each is rounded by itself,
so codes, powers of two and fp32 moments are compared bit for bit); the parameters in 64 bits from those."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2209_13258_amd as osdp

pytestmark = pytest.mark.gpu

M32 = 0xFFFFFFFF
EPS24 = 2.0 ** -24
LENGTHS = [0, 1, 2, 127, 128, 129, 1000, 2047, 2048, 2049, 4096, 5000, 70001]


def mix(x):
    x = (x * 0x9E3779B1) & M32
    x = x ^ (x >> 15)
    x = (x * 0x2C1B3C6D) & M32
    return x ^ (x >> 13)


def randoms(n, seed, step, place):
    """16 random bits each for m, v and a bf16 parameter of elements 0 .. n - 1."""
    key = mix(mix(mix(mix(seed & M32) ^ (seed >> 32)) ^ (step & M32)) ^ place)
    h = mix((np.arange(n, dtype=np.uint64) + mix(key)) & M32)
    return h & 0xFFFF, h >> 16, ((h * 0x297A2D39) & M32) >> 16


def bits(x):
    return np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.int64)


def encode(x, r16, top, low):
    """(codes, exponents of the blocks) of fp32 values, from the format's definition."""
    n = x.size
    a = np.abs(x)
    padded = np.zeros(-(-n // 128) * 128, np.float32)
    padded[:n] = a
    most = bits(padded).reshape(-1, 128).max(axis=1)
    b = np.where(most == 0, 0, np.maximum((most + 0xFFFFF) >> 23, low))
    b = np.where(most >= 0x7F800000, 255, b)
    least = np.repeat(b - (top - 1), 128)[:n]
    e = np.maximum(bits(a) >> 23, least)
    with np.errstate(invalid="ignore"):
        units = np.ldexp(a.astype(np.float64), (130 - e).astype(np.int64))      # exact
        total = (units + r16.astype(np.float64) / 65536).astype(np.float32)     # one rounding, as in fp32
        q = np.floor(np.nan_to_num(total)).astype(np.int64)
    code = (e - least) * 8 + q
    if top == 31:
        code = np.where((a > 0) & (code == 0), 1, code)
    else:
        code = code | ((bits(x) >> 31) << 7)
    per = np.repeat(b, 128)[:n]
    return np.where((per == 0) | (per == 255), 0, code).astype(np.uint8), b.astype(np.uint8)


def decode(code, b, top):
    c = code.astype(np.int64)
    mag = c & 127 if top == 15 else c
    per = np.repeat(b.astype(np.int64), 128)[:c.size]
    E, f = mag >> 3, mag & 7
    v = np.where(E > 0, np.ldexp(1 + f / 8.0, (per - 127 - top + E)), np.ldexp(f / 8.0, per - 126 - top))
    v = np.where(per == 0, 0.0, np.where(per == 255, np.nan, v))
    return (np.where(c > 127, -v, v) if top == 15 else v).astype(np.float32)


class Case:
    """Tensors of the given lengths side by side in flat buffers, `gap` elements apart, and what they should become."""

    def __init__(self, lengths, state=32, param="master", grad="bf16", gap=0, seed=0, zero=False, decay=0.1):
        g = np.random.default_rng(seed)
        self.lengths, self.state, self.param = lengths, state, param
        self.start, at = [], gap
        for n in lengths:
            self.start.append(at)
            at += n + gap if gap % 128 else -(-n // 128) * 128 + gap
        total = at + 128
        spread = np.exp(2 * np.repeat(g.standard_normal(-(-total // 64)), 64)[:total])
        f32 = lambda x: torch.from_numpy(x.astype(np.float32)).cuda()  # noqa: E731
        self.grad = f32(g.standard_normal(total) * 1e-3 * spread).to(torch.bfloat16 if grad == "bf16" else torch.float32)
        self.weight = f32(g.standard_normal(total) * 0.02)
        self.p = self.weight.clone() if param == "f32" else self.weight.to(torch.bfloat16)
        self.master = self.weight.clone() if param == "master" else None
        z = 0.0 if zero else 1.0
        m, v = g.standard_normal(total) * 3e-4 * spread * z, (0.5 + g.random(total)) * 1e-6 * spread ** 2 * z
        self.exps = None
        if state == 32:
            self.m, self.v = f32(m), f32(v)
        else:
            self.m = torch.from_numpy(g.integers(0, 256, total).astype(np.uint8)).cuda()
            self.v = torch.from_numpy(g.integers(0, 256, total).astype(np.uint8)).cuda()
            self.exps = []
            for i, n in enumerate(lengths):
                a = self.start[i]
                mc, mb = encode(m[a:a + n].astype(np.float32), np.full(n, 32768), 15, 32)
                vc, vb = encode(v[a:a + n].astype(np.float32), np.full(n, 32768), 31, 48)
                self.m[a:a + n] = torch.from_numpy(mc).cuda()
                self.v[a:a + n] = torch.from_numpy(vc).cuda()
                self.exps.append(torch.from_numpy(np.stack([mb, vb], 1).copy()).cuda())
        self.decay = [decay * (i % 3) for i in range(len(lengths))]
        self.flat = {k: t for k, t in dict(params=self.p, grads=self.grad, masters=self.master, m=self.m, v=self.v).items() if t is not None}
        self.before = {k: t.clone() for k, t in self.flat.items()}
        self.exps_before = [e.clone() for e in self.exps] if self.exps else None
        self.views = {k: [t[a:a + n] for a, n in zip(self.start, lengths)] for k, t in self.flat.items()}
        self.table = osdp.AdamWTable(exps=self.exps, weight_decay=self.decay, **self.views)

    def part(self, name, i, before=False):
        t = (self.before if before else self.flat)[name][self.start[i]:self.start[i] + self.lengths[i]]
        return t.float().cpu().numpy() if t.dtype != torch.uint8 else t.cpu().numpy()

    def check(self, lr, b1, b2, eps, step, seed, coef=1.0):
        torch.cuda.synchronize()
        one = np.float32
        for i, n in enumerate(self.lengths):
            if n == 0:
                continue
            g = self.part("grads", i, True) * one(coef)
            if self.state == 32:
                m, v = self.part("m", i, True), self.part("v", i, True)
            else:
                eb = self.exps_before[i].cpu().numpy()
                m, v = decode(self.part("m", i, True), eb[:, 0], 15), decode(self.part("v", i, True), eb[:, 1], 31)
            m1 = m * one(b1) + g * one(1 - b1)
            v1 = v * one(b2) + (g * g) * one(1 - b2)
            um, uv, up = randoms(n, seed, step, i)
            if self.state == 32:
                assert np.array_equal(self.part("m", i), m1) and np.array_equal(self.part("v", i), v1), f"tensor {i}: moments"
            else:
                e = self.exps[i].cpu().numpy()
                for name, x, u, top, low, col in (("m", m1, um, 15, 32, 0), ("v", v1, uv, 31, 48, 1)):
                    code, b = encode(x, u, top, low)
                    assert np.array_equal(e[:, col], b), f"tensor {i}: {name}'s powers of two"
                    assert np.array_equal(self.part(name, i), code), f"tensor {i}: {name}'s codes"
            source = self.part("masters" if self.param == "master" else "params", i, True).astype(np.float64)
            update = lr / (1 - b1 ** step) * m1.astype(np.float64) / (np.sqrt(v1.astype(np.float64) / (1 - b2 ** step)) + eps)
            decay = lr * self.decay[i] * source
            p1 = source - decay - update
            # Roundings on the way to p, in half steps of fp32 (2^-24 of the value each): rate, root, m * rate, the fused
            # product and sum of the denominator, the fused sum (1 each), square root and reciprocal (an ulp, so 2 each),
            # 9 on the update; lr, the tensor's decay, their product and its own with p, the sum, 5 on the decay; 1 on p.
            tol = EPS24 * (np.abs(p1) + 10 * np.abs(update) + 6 * np.abs(decay)) * 1.01
            if self.param == "master":
                got = self.part("masters", i)
                assert (np.abs(got - p1) <= tol).all(), f"tensor {i}: off by {np.abs(got - p1).max():.3e}"
                nearest = torch.from_numpy(got).to(torch.bfloat16).float().numpy()
                assert np.array_equal(self.part("params", i), nearest), f"tensor {i}: parameters are not the rounded masters"
            elif self.param == "f32":
                got = self.part("params", i)
                assert (np.abs(got - p1) <= tol).all(), f"tensor {i}: off by {np.abs(got - p1).max():.3e}"
            else:
                got = self.part("params", i).astype(np.float64)
                grid = np.exp2(np.floor(np.log2(np.maximum(np.abs(p1), 1e-38))) - 7)
                lo = np.floor((np.abs(p1) - tol) / grid + up / 65536.0) * grid
                hi = np.floor((np.abs(p1) + tol) / grid + up / 65536.0) * grid
                # The kernel's fp32 value lies within tol of p1, and rounding (the sum of its size and a number, cut) keeps order:
                # the result lies between what the two ends of that range give.  These are the same or neighbours but where
                # a weight and its update all but cancel and tol is many steps of the small result.
                ok = (np.abs(got) >= lo) & (np.abs(got) <= hi)
                edge = np.abs(np.abs(p1) / np.exp2(np.round(np.log2(np.maximum(np.abs(p1), 1e-38)))) - 1) < 1e-5  # at a power of two the grid changes
                assert (ok | edge).all(), f"tensor {i}: {int((~(ok | edge)).sum())} parameters rounded otherwise"
        for k, t in self.flat.items():  # what lies between the tensors is left as it was, and so are the gradients
            keep = torch.ones(t.numel(), dtype=torch.bool, device="cuda")
            if k != "grads":
                for a, n in zip(self.start, self.lengths):
                    keep[a:a + n] = False
            same = t.view(torch.uint8).view(t.numel(), -1) == self.before[k].view(torch.uint8).view(t.numel(), -1)
            assert same[keep].all(), f"{k}: something outside the tensors was written"


@pytest.mark.parametrize("gap", [0, 128, 3])
@pytest.mark.parametrize("state,param,grad", [(32, "master", "bf16"), (32, "f32", "f32"), (32, "bf16", "bf16"), (8, "master", "bf16"),
                                              (8, "bf16", "bf16"), (8, "f32", "f32"), (8, "master", "f32"), (32, "bf16", "f32"),
                                              (32, "f32", "bf16"), (8, "f32", "bf16"), (8, "bf16", "f32"), (32, "master", "f32")])
def test_step_against_the_formulas(state, param, grad, gap):
    print("adamw", state, param, grad, "gap", gap, flush=True)
    c = Case(LENGTHS, state, param, grad, gap, seed=gap)
    for step in (7,):
        osdp.osdp_adamw_step(c.table, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=step, seed=(5 << 40) + 11)
        c.check(1e-3, 0.9, 0.95, 1e-8, step, (5 << 40) + 11)


@pytest.mark.parametrize("state", [32, 8])
def test_first_step_from_zero_moments(state):
    c = Case([300, 2048], state, "master", zero=True)
    if state == 8:
        for t in [c.m, c.v, *c.exps]:
            t.zero_()
        c.before["m"].zero_()
        c.before["v"].zero_()
        c.exps_before = [e.clone() for e in c.exps]
    osdp.osdp_adamw_step(c.table, lr=1e-2, step=1, seed=3)
    c.check(1e-2, 0.9, 0.999, 1e-8, 1, 3)


@pytest.mark.parametrize("state", [32, 8])
def test_many_tensors_take_several_launches(state):
    g = np.random.default_rng(1)
    lengths = [int(n) for n in g.integers(0, 400, 150)]
    lengths[3] = lengths[60] = 0
    c = Case(lengths, state, "master")
    osdp.osdp_adamw_step(c.table, lr=1e-3, step=2, seed=9)
    c.check(1e-3, 0.9, 0.999, 1e-8, 2, 9)


def test_no_tensors_and_empty_ones():
    for lengths in ([], [0], [0, 0, 0]):
        t = osdp.AdamWTable(params=[torch.empty(n, device="cuda") for n in lengths], grads=[torch.empty(n, device="cuda") for n in lengths],
                            m=[torch.empty(n, device="cuda") for n in lengths], v=[torch.empty(n, device="cuda") for n in lengths])
        osdp.osdp_adamw_step(t, lr=1e-3)
        out = torch.full((1,), 5.0, dtype=torch.float64, device="cuda")
        ws = torch.empty(256, dtype=torch.uint8, device="cuda")
        osdp.osdp_adamw_grad_sumsq(t, out, ws, accumulate=True)
        assert out.item() == 5.0
        osdp.osdp_adamw_grad_sumsq(t, out, ws)
        assert out.item() == 0.0


@pytest.mark.parametrize("param,state", [("bf16", 8), ("master", 32)])
def test_a_large_step_whose_tensors_end_anywhere(param, state):
    """Enough elements for a workgroup to take several tiles one after another, across the ends of tensors short and long."""
    c = Case([5000003, 2047, 3000000, 1, 0, 4700001, 64, 129, 130000], state, param, seed=8)
    osdp.osdp_adamw_step(c.table, lr=1e-3, step=7, seed=12)
    c.check(1e-3, 0.9, 0.999, 1e-8, 7, 12)


def test_the_factor_that_clips_is_the_quotient():
    """m is the factor itself after a step over gradients of 1 with beta1 = 0."""
    g = np.random.default_rng(4)
    sums = list(10.0 ** g.uniform(-290, 300, 150)) + [1e-300, 1e308, 1.0, 4.0, 1.0 + 2.0 ** -52, 2.0]
    m = torch.zeros(8, device="cuda")
    table = osdp.AdamWTable(params=[torch.zeros(8, device="cuda")], grads=[torch.ones(8, device="cuda")], m=[m], v=[torch.zeros(8, device="cuda")])
    for s in sums:
        for bound in (np.sqrt(s) * g.uniform(1e-3, 1.0), np.sqrt(s) * 10.0 ** g.uniform(-30, 0), 2.0 * np.sqrt(s), 1.0):
            total = torch.tensor([s], dtype=torch.float64, device="cuda")
            osdp.osdp_adamw_step(table, lr=0.0, beta1=0.0, step=1, grad_sumsq=total, max_norm=float(bound))
            q = float(bound) / np.sqrt(s) if np.sqrt(s) > bound else 1.0
            with np.errstate(over="ignore", under="ignore"):  # (its own error, below 2^-40, may turn a rounding's tie)
                ends = np.float32(q * (1 - 2.0 ** -40)), np.float32(q * (1 + 2.0 ** -40))
            got = m[3].item()
            assert ends[0] <= got <= ends[1], (s, bound, got, q)


@pytest.mark.parametrize("factor", [0.5, 1.0, 7.0])
def test_clipping_by_the_norm(factor):
    """The norm found by the one call is what the other clips by; a norm below the bound changes nothing."""
    c = Case([5000, 129], 32, "f32", "f32")
    ws = torch.empty(osdp.osdp_adamw_grad_sumsq_workspace_bytes(c.table), dtype=torch.uint8, device="cuda")
    sumsq = torch.empty(1, dtype=torch.float64, device="cuda")
    osdp.osdp_adamw_grad_sumsq(c.table, sumsq, ws)
    norm = float(sumsq.sqrt())
    osdp.osdp_adamw_step(c.table, lr=1e-3, step=4, grad_sumsq=sumsq, max_norm=norm / factor)
    coef = (norm / factor) / norm if norm > norm / factor else 1.0
    c.check(1e-3, 0.9, 0.999, 1e-8, 4, 0, coef=np.float32(coef))


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_no_number_leaves_everything(bad, state):
    c = Case([700, 2048], state, "master")
    c.grad[c.start[1] + 5] = bad
    ws = torch.empty(osdp.osdp_adamw_grad_sumsq_workspace_bytes(c.table), dtype=torch.uint8, device="cuda")
    sumsq = torch.empty(1, dtype=torch.float64, device="cuda")
    osdp.osdp_adamw_grad_sumsq(c.table, sumsq, ws)
    assert not np.isfinite(sumsq.item())
    for max_norm in (0.0, 1.0):
        osdp.osdp_adamw_step(c.table, lr=1e-3, step=4, grad_sumsq=sumsq, max_norm=max_norm)
    torch.cuda.synchronize()
    for k in ("params", "masters", "m", "v"):
        assert torch.equal(c.flat[k], c.before[k]), k
    for e, old in zip(c.exps or [], c.exps_before or []):
        assert torch.equal(e, old)


def test_numbers_that_are_none_stay_in_their_block():
    """Without a norm to go by, a NaN gradient makes NaN of its own element (fp32) or of its own block of moments (8 bits)."""
    for state in (32, 8):
        c = Case([1024], state, "f32", "f32")
        c.grad[c.start[0] + 300] = float("nan")
        osdp.osdp_adamw_step(c.table, lr=1e-3, step=3)
        p = c.p[c.start[0]:c.start[0] + 1024]
        assert torch.isnan(p).nonzero().flatten().tolist() == [300]
        if state == 8:
            assert (c.exps[0][:, 0] == 255).nonzero().flatten().tolist() == [2]
            out = [torch.empty(1024, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            osdp.osdp_adamw_state_values(c.table, out[:1], out[1:])
            for o in out:
                assert torch.isnan(o[256:384]).all() and torch.isfinite(o[:256]).all() and torch.isfinite(o[384:]).all()


@pytest.mark.parametrize("gap", [0, 3])
@pytest.mark.parametrize("param,grad", [("bf16", "bf16"), ("bf16", "f32"), ("master", "f32"), ("f32", "f32"), ("master", "bf16")])
def test_not_a_number_of_any_sign_and_payload(param, grad, gap):
    """In 8 bits: the element's parameter is NaN, its block's powers say so and its codes are zeros; all else is as without it."""
    c = Case([4096, 700], 8, param, grad, gap, seed=6)
    at = [5, 128 + 127, 1280, 2047, 3500]
    patterns = [0xFFFFFFFF, 0x7FFFFFFF, 0xFF800001, 0xFFC00000, 0x7FA00000]
    whole = c.grad.view(torch.int32 if grad == "f32" else torch.int16)
    for i, b in zip(at, patterns):
        if grad == "bf16":
            b = (b >> 16) | (1 if b & 0xFFFF else 0)
        whole[c.start[0] + i] = b - (1 << (32 if grad == "f32" else 16)) if b >> (31 if grad == "f32" else 15) else b
    assert c.grad.isnan().sum() == len(at)
    c.before["grads"] = c.grad.clone()
    osdp.osdp_adamw_step(c.table, lr=1e-3, step=3, seed=2)
    torch.cuda.synchronize()
    m, v, e = c.part("m", 0), c.part("v", 0), c.exps[0].cpu().numpy()
    blocks = sorted({i // 128 for i in at})
    assert sorted(np.flatnonzero(e[:, 0] == 255)) == blocks and sorted(np.flatnonzero(e[:, 1] == 255)) == blocks
    for b in blocks:
        assert not m[b * 128:b * 128 + 128].any() and not v[b * 128:b * 128 + 128].any()
    for name in ("params", "masters") if param == "master" else ("params",):
        assert sorted(np.flatnonzero(np.isnan(c.part(name, 0)))) == at
        assert not np.isnan(c.part(name, 1)).any()


@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("state,param", [(8, "bf16"), (32, "bf16"), (8, "master"), (32, "master"), (8, "f32"), (32, "f32")])
def test_a_rate_that_is_not_a_number(state, param, grad):
    """Whatever its sign and payload every parameter becomes NaN, none a number, and the moments are those of any rate."""
    for pattern in (0x7FFFFFFF, 0xFFFFFFFF, 0x7F800001, 0xFFC00000):
        rate = torch.tensor([pattern - (1 << 32 if pattern >> 31 else 0)], dtype=torch.int64, device="cuda").to(torch.int32).view(torch.float32)
        c, other = (Case([3000, 129], state, param, grad, gap=1, seed=9) for _ in range(2))
        osdp.osdp_adamw_step(c.table, lr=0.0, lr_device=rate, step=3, seed=2)
        osdp.osdp_adamw_step(other.table, lr=1e-3, step=3, seed=2)
        torch.cuda.synchronize()
        for name in ("params", "masters") if param == "master" else ("params",):
            for i in range(2):
                assert np.isnan(c.part(name, i)).all(), (hex(pattern), name, i)
        for name in ("m", "v"):
            assert torch.equal(c.flat[name], other.flat[name])


@pytest.mark.parametrize("gap", [0, 5])
def test_state_values_are_the_codes_values(gap):
    c = Case([1, 127, 128, 300, 4096, 0, 2051], 8, "bf16", gap=gap)
    total = c.m.numel()
    outs = {k: torch.full((total,), 7.0, dtype=torch.bfloat16, device="cuda") for k in "mv"}
    osdp.osdp_adamw_state_values(c.table, *[[outs[k][a:a + n] for a, n in zip(c.start, c.lengths)] for k in "mv"])
    torch.cuda.synchronize()
    for k, top, col in (("m", 15, 0), ("v", 31, 1)):
        left = torch.ones(total, dtype=torch.bool)
        for i, (a, n) in enumerate(zip(c.start, c.lengths)):
            want = decode(c.part(k, i), c.exps[i].cpu().numpy()[:, col], top)
            assert np.array_equal(outs[k][a:a + n].float().cpu().numpy(), want)
            left[a:a + n] = False
        assert (outs[k].cpu()[left] == 7.0).all()


def test_every_code_of_the_format_survives_a_step_that_changes_nothing():
    """beta = 0 and lr = 0 with gradients that are m's values: they lie on the grid, so that no random number moves them."""
    codes = np.arange(256)
    for b in (32, 100, 127, 200, 254):
        block = np.concatenate([codes[:128], codes[128:]])
        values = decode(block.astype(np.uint8), np.array([b, b], np.uint8), 15)
        g = torch.from_numpy(values).cuda()
        z = lambda t: torch.zeros(256, dtype=t, device="cuda")  # noqa: E731
        p, m, v, e = torch.zeros(256, device="cuda"), z(torch.uint8), z(torch.uint8), torch.zeros(4, dtype=torch.uint8, device="cuda")
        t = osdp.AdamWTable(params=[p], grads=[g], m=[m], v=[v], exps=[e])
        osdp.osdp_adamw_step(t, lr=0.0, beta1=0.0, beta2=0.0, step=1, seed=b)
        want = np.where(block == 128, 0, block)  # (m is 0 * 0 plus the value: of -0 that is 0)
        assert m.cpu().numpy().tolist() == want.tolist(), b
        assert e.cpu().numpy()[::2].tolist() == [b, b]
        with np.errstate(over="ignore"):
            squares = values * values
        if np.isinf(squares).any():  # (of the largest blocks: no numbers, and the block says so)
            assert e.cpu().numpy()[1::2].tolist() == [255, 255]
        else:
            assert (v.cpu().numpy()[squares > 0] > 0).all()


def test_stochastic_rounding_keeps_the_mean():
    """A weight that moves by a thirtieth of its rounding step, many times: the mean of many of them follows.  (The standard deviation of a
    step's rounding is at most half a step of 2^-8 here, of the mean over 2^16 elements and 30 steps 2^-9 sqrt(30) / 2^8.)"""
    n, steps, lr = 1 << 16, 30, 2.0 ** -8 / 30
    p = torch.full((n,), 1.5, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(n, device="cuda")
    m, v, e = (torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, n, 2 * n // 128))
    t = osdp.AdamWTable(params=[p], grads=[g], m=[m], v=[v], exps=[e])
    for k in range(steps):
        osdp.osdp_adamw_step(t, lr=lr, beta1=0.0, beta2=0.0, step=k + 1, seed=77)
    moved = 1.5 - p.double().mean().item()
    assert abs(moved - steps * lr) < 6 * 2.0 ** -9 * 30 ** 0.5 / 2 ** 8 + steps * lr * 1e-5


def test_moments_in_8_bits_follow_those_in_32():
    """v decays by 5 % a step, less than half of its grid's 12.5 %: nearest rounding would keep it where it is for ever.  After 20
    steps of zero gradients the mean over a block's 0.95^20 is exact, and each rounding adds at most (grid / 2)^2 of variance."""
    n, steps = 1 << 15, 20
    g = torch.zeros(n, device="cuda")
    p = torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    e = torch.zeros(2 * n // 128, dtype=torch.uint8, device="cuda")
    t = osdp.AdamWTable(params=[p], grads=[torch.full((n,), 0.37, device="cuda")], m=[m], v=[v], exps=[e])
    osdp.osdp_adamw_step(t, lr=0.0, beta1=0.0, beta2=0.0, step=1, seed=1)
    t.set_grads([g])
    for k in range(steps):
        osdp.osdp_adamw_step(t, lr=0.0, beta1=0.95, beta2=0.95, step=k + 2, seed=1)
    out = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    osdp.osdp_adamw_state_values(t, out[:1], out[1:])
    for got, start in ((out[0], 0.37), (out[1], 0.37 ** 2)):
        want = start * 0.95 ** steps
        # relative standard deviation of the mean: sqrt(steps + 1) roundings of at most 1/16 each (the steps are 1/8 to 1/16 of a value), over sqrt(n)
        assert abs(got.double().mean().item() / want - 1) < 6 * (steps + 1) ** 0.5 / 16 / n ** 0.5


def test_the_same_call_gives_the_same_bits_and_another_seed_others():
    def run(seed, step=5):
        c = Case([3000, 128], 8, "bf16")
        osdp.osdp_adamw_step(c.table, lr=1e-3, step=step, seed=seed)
        torch.cuda.synchronize()
        return [c.p.clone(), c.m.clone(), c.v.clone()]
    a, b, other, later = run(1), run(1), run(2), run(1, 6)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert not torch.equal(a[1], other[1]) and not torch.equal(a[2], later[2])


@pytest.mark.parametrize("state", [32, 8])
def test_captured_step_takes_step_and_rate_from_the_device(state):
    """A graph of norm and step, replayed with the program's own work between, against eager calls."""
    def make():
        c = Case([3000, 129], state, "master")
        ws = torch.zeros(osdp.osdp_adamw_grad_sumsq_workspace_bytes(c.table), dtype=torch.uint8, device="cuda")
        return c, ws, torch.zeros(1, dtype=torch.float64, device="cuda")
    eager, ws, sumsq = make()
    graph, gws, gsum = make()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    rate = torch.zeros(1, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        osdp.osdp_adamw_grad_sumsq(graph.table, gsum, gws, stream=stream)
        osdp.osdp_adamw_step(graph.table, lr=0.0, step_device=step, lr_device=rate, grad_sumsq=gsum, max_norm=0.01, seed=4, stream=stream)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for k in range(1, 5):
        lr = 2.0 ** -9 / k
        new = torch.randn(eager.grad.shape, generator=gen, device="cuda").mul_(1e-3).to(torch.bfloat16)
        eager.grad.copy_(new)
        graph.grad.copy_(new)
        step.fill_(k)
        rate.fill_(lr)
        gws.fill_(255)  # nothing of the workspace is kept from one call to the next
        torch.cuda.synchronize()
        g.replay()
        osdp.osdp_adamw_grad_sumsq(eager.table, sumsq, ws)
        osdp.osdp_adamw_step(eager.table, lr=float(np.float32(lr)), step=k, grad_sumsq=sumsq, max_norm=0.01, seed=4)
        torch.cuda.synchronize()
        assert torch.equal(sumsq, gsum)
        for name in ("params", "masters", "m", "v"):
            assert torch.equal(eager.flat[name], graph.flat[name]), (k, name)


@pytest.mark.parametrize("lengths", [[3000, 129], [12500003, 100001, 1]])
@pytest.mark.parametrize("state,param", [(8, "bf16"), (32, "bf16"), (8, "f32"), (32, "f32"), (8, "master"), (32, "master")])
def test_step_and_rate_on_the_device_one_by_one(state, param, lengths):
    """Either alone and both, in a graph that is replayed, against eager calls with the same numbers from the host; what is below 1 counts as step 1.
    The longer list has enough tiles for a workgroup of the bf16 form in 8 bits to take four."""
    host, dev = (Case(lengths, state, param, gap=1, seed=5) for _ in range(2))
    step, rate = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    stream = torch.cuda.Stream()
    kwargs = dict(beta1=0.9, beta2=0.95, seed=21)
    for which in ("step", "rate", "both"):
        on_device = dict(step_device=step if which != "rate" else None, lr_device=rate if which != "step" else None)
        at = {"step": 1, "rate": 6, "both": 1}[which]  # (what the graph holds: a step that is not read, and one that is)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            osdp.osdp_adamw_step(dev.table, lr=2.0 ** -10 if which == "step" else 0.0, step=at, stream=stream, **on_device, **kwargs)
        for t in (-3, 0, 1, 2, 1000, 10 ** 7) if len(lengths) == 2 else (2, 1000):
            lr = float(np.float32(3e-4 / max(t, 1) ** 0.25))
            step.fill_(t)
            rate.fill_(lr)
            torch.cuda.synchronize()
            g.replay()
            osdp.osdp_adamw_step(host.table, lr=2.0 ** -10 if which == "step" else lr, step=6 if which == "rate" else max(t, 1), **kwargs)
            torch.cuda.synchronize()
            for name, x in host.flat.items():
                assert torch.equal(x, dev.flat[name]), (which, t, name)
            for a, b in zip(host.exps or [], dev.exps or []):
                assert torch.equal(a, b), (which, t)


def test_streams_of_the_caller():
    a, b = Case([200000], 32, "master", seed=1), Case([200000], 8, "bf16", seed=2)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    osdp.osdp_adamw_step(a.table, lr=1e-3, step=7, seed=1, stream=sa)
    osdp.osdp_adamw_step(b.table, lr=1e-3, step=7, seed=2, stream=sb)
    sa.synchronize()
    a.check(1e-3, 0.9, 0.999, 1e-8, 7, 1)
    sb.synchronize()
    b.check(1e-3, 0.9, 0.999, 1e-8, 7, 2)


def test_more_elements_than_32_bits_count():
    """Places beyond 2^31 and 2^32: their own numbers, powers of two and random bits, and no others'."""
    n, step, seed = (1 << 32) + 4096 + 77, 3, 19
    print("adamw", n, "elements", flush=True)
    z = lambda t, k=n: torch.zeros(k, dtype=t, device="cuda")  # noqa: E731
    p, g, m, v, e = z(torch.bfloat16), z(torch.bfloat16), z(torch.uint8), z(torch.uint8), z(torch.uint8, 2 * -(-n // 128))
    starts = [0, (1 << 31) - 256, (1 << 32) - 256, n - 333]
    rng = np.random.default_rng(4)
    parts = {}
    for a in starts:
        a -= a % 128
        k = min(512, n - a)
        parts[a] = torch.from_numpy(rng.standard_normal((2, k)).astype(np.float32)).to(torch.bfloat16)
        g[a:a + k], p[a:a + k] = parts[a][0].cuda(), parts[a][1].cuda()
    table = osdp.AdamWTable(params=[p], grads=[g], m=[m], v=[v], exps=[e])
    sumsq, ws = z(torch.float64, 1), z(torch.uint8, osdp.osdp_adamw_grad_sumsq_workspace_bytes(table))
    osdp.osdp_adamw_grad_sumsq(table, sumsq, ws)
    osdp.osdp_adamw_step(table, lr=1e-2, beta1=0.5, beta2=0.5, step=step, seed=seed)
    torch.cuda.synchronize()
    want = sum(float((x[0].double() ** 2).sum()) for x in parts.values())
    assert abs(sumsq.item() / want - 1) < 2.0 ** -39
    one, touched = np.float32, 0
    for a, x in parts.items():
        k = x.shape[1]
        key = mix(mix(mix(mix(mix(seed) ^ 0) ^ step) ^ 0) ^ (a >> 32))
        h = mix((np.arange(a, a + k, dtype=np.uint64) + key) & M32)   # (none of the parts crosses 2^32 within itself ...
        if (a >> 32) != ((a + k - 1) >> 32):                          # ... but one, whose second half counts anew)
            key2 = mix(mix(mix(mix(mix(seed) ^ 0) ^ step) ^ 0) ^ ((a >> 32) + 1))
            h2 = mix((np.arange(a, a + k, dtype=np.uint64) + key2) & M32)
            h = np.where(np.arange(a, a + k) >> 32 == a >> 32, h, h2)
        gr = x[0].float().numpy()
        m1, v1 = gr * one(0.5), (gr * gr) * one(0.5)
        for name, val, r16, top, low, dev, col in (("m", m1, h & 0xFFFF, 15, 32, m, 0), ("v", v1, h >> 16, 31, 48, v, 1)):
            code, b = encode(val, r16, top, low)
            assert np.array_equal(dev[a:a + k].cpu().numpy(), code), (name, a)
            assert np.array_equal(e[2 * (a // 128):2 * (a // 128) + 2 * b.size].cpu().numpy()[col::2], b), (name, a)
        touched += int((m[a:a + k] != 0).sum())
    assert int((m != 0).sum()) == touched, "moments outside the parts with gradients were written"


@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,gap", [([1], 0), ([7, 0, 4097], 3), (LENGTHS, 0), ([3000001], 1), ([40] * 130, 0)])
def test_sum_of_squares(grad, lengths, gap):
    print("sumsq", grad, lengths[:4], gap, flush=True)
    c = Case(lengths, 32, "f32", grad, gap)
    c.grad[c.start[0]] = 3e30  # its square is no fp32 number
    total = sum(float((c.grad[a:a + n].double() ** 2).sum()) for a, n in zip(c.start, lengths))
    ws = torch.full((osdp.osdp_adamw_grad_sumsq_workspace_bytes(c.table),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda")
    osdp.osdp_adamw_grad_sumsq(c.table, out, ws)
    first = out.item()
    # either side: chains of fewer than 2^13 additions, all of one sign, each off by at most 2^-53 of the sum
    assert abs(first / total - 1) < 2.0 ** -39
    osdp.osdp_adamw_grad_sumsq(c.table, out, ws, accumulate=True)
    assert out.item() == 2 * first
    osdp.osdp_adamw_grad_sumsq(c.table, out, ws)
    assert out.item() == first


@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[9000], [70000], [5, 4099, 30001], [1 << 20, 300001], [5000003, 2047, 1, 4700001, 129]])
def test_sum_of_squares_at_any_alignment(grad, lengths):
    """The order of the sum depends on the lengths alone: the same gradients give the same bits wherever they lie, in tensors of their own and packed
    side by side, in one launch, in two, and in runs of four tiles."""
    kind = torch.bfloat16 if grad == "bf16" else torch.float32
    # (of magnitudes far enough apart that 53 bits do not hold their squares' sums exactly, whatever their order)
    values = [torch.randn(2, n, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda") for n in lengths]
    values = [(x[0] * torch.exp2(8 * x[1])).to(kind) for x in values]
    total = sum(float((x.double() ** 2).sum()) for x in values)
    out = torch.full((1,), float("nan"), dtype=torch.float64, device="cuda")
    sums = {}
    for first in (0, 1, 2, 3, 8):
        for packed in (False, True):
            grads = []
            if packed:
                flat = torch.full((first + sum(lengths) + 8,), 1e4, dtype=kind, device="cuda")
                at = first
                for x in values:
                    grads.append(flat[at:at + x.numel()].copy_(x))
                    at += x.numel()
            else:
                grads = [torch.full((first + x.numel() + 8,), 1e4, dtype=kind, device="cuda")[first:first + x.numel()].copy_(x) for x in values]
            table = osdp.AdamWTable(grads=grads)
            ws = torch.full((max(8, osdp.osdp_adamw_grad_sumsq_workspace_bytes(table)),), 255, dtype=torch.uint8, device="cuda")
            osdp.osdp_adamw_grad_sumsq(table, out, ws)
            sums[first, packed] = out.item()
    # either side: chains of fewer than 2^13 additions, all of one sign, each off by at most 2^-53 of the sum
    assert abs(sums[0, False] / total - 1) < 2.0 ** -39
    assert len(set(sums.values())) == 1, sums


def test_table_refusals():
    t = lambda n, d=torch.float32: torch.zeros(n, dtype=d, device="cuda")  # noqa: E731
    bad = [dict(grads=[t(4)], params=[t(5)]), dict(grads=[t(4)], params=[t(4), t(4)]), dict(grads=[t(4, torch.float16)]),
           dict(grads=[t(8)[::2]]), dict(grads=[t(4)], m=[t(4)], v=[t(4, torch.uint8)]), dict(grads=[t(4), t(4, torch.bfloat16)]),
           dict(grads=[t(4)], m=[t(4, torch.uint8)], v=[t(4, torch.uint8)]), dict(grads=[t(4)], weight_decay=[0.1, 0.2]),
           dict(grads=[t(300)], m=[t(300, torch.uint8)], v=[t(300, torch.uint8)], exps=[t(5, torch.uint8)])]
    for kw in bad:
        with pytest.raises(osdp.OsdpError) as e:
            osdp.AdamWTable(**kw)
        assert e.value.status == osdp.binding.OSDP_ERR_INVALID_ARG
    table = osdp.AdamWTable(grads=[t(4)], params=[t(4)], m=[t(4)], v=[t(4)])
    for kw in (dict(grad_sumsq=t(1)), dict(step_device=t(1)), dict(lr_device=t(2)), dict(max_norm=1.0)):
        with pytest.raises(osdp.OsdpError):
            osdp.osdp_adamw_step(table, lr=1e-3, **kw)
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_adamw_state_values(table, [t(4, torch.bfloat16)], [t(4, torch.bfloat16)])
    with pytest.raises(osdp.OsdpError):
        table.set_grads([t(5)])


def test_tables_whose_tensors_share_memory():
    t = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    p, g, flat = t(64), t(64), t(256)
    piece = lambda i, n=64: flat[i:i + n]  # noqa: E731
    for kw in (dict(params=[p, p], grads=[g, t(64)], m=[t(64), t(64)], v=[t(64), t(64)]),            # listed twice
               dict(params=[p], grads=[p], m=[t(64)], v=[t(64)]), dict(params=[p], grads=[g], m=[p], v=[t(64)]),
               dict(params=[piece(0)], grads=[g], m=[piece(63)], v=[piece(128)]),                     # by one element
               dict(params=[piece(0)], grads=[piece(191)], m=[piece(64)], v=[piece(128)])):
        with pytest.raises(osdp.OsdpError, match="share memory"):
            osdp.AdamWTable(**kw)
    osdp.AdamWTable(params=[piece(0)], grads=[piece(192)], m=[piece(64)], v=[piece(128)])             # side by side
    osdp.AdamWTable(params=[p, t(64)], grads=[g, g], m=[t(64), t(64)], v=[t(64), t(64)])              # read twice
    osdp.AdamWTable(grads=[g, g])
