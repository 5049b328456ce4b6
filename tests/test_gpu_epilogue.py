"""The operator with bias, activation and residual, and its backward pass, against the formulas in 64 bits.

Tolerances.  A value rounded to bf16 is off by 2^-8 of it at most (half a step).  The sum in fp32 over K up to 32768 products stays
below 1e-3 of the outputs' root mean square, as the other products' tests take it; an activation passes that on times its slope, at
most 1.13, and adds 2^-15 of its own value.  Y = act + R: 2^-8 |Y| + 2^-15 |act| + 1.13e-3 rms(z).  dZ = dY act'(Z): 2^-8 |dZ| + 2^-15 |dY|
(the slope is off by 2^-15, by itself), and 2^-23 |dZ| for the product in fp32.  db: each term is off by 2^-15 |dY| + 2^-23 |dZ|, the sum of T of them in
fp32, by partial sums, by T 2^-24 of the sum of magnitudes at most, then half a step of its type.  dX and dW are products of the dZ that
was stored: 2^-8 of them and 1e-3 of their root mean square, and bit by bit those of the product's own backward pass where neither
runs in parts of its reduction."""
from __future__ import annotations

import threading

import pytest
import torch

import epilogue_reference as R
import gpu_harness as H
import paper_2209_13258_amd as osdp

pytestmark = pytest.mark.gpu
ACTS = {n: getattr(osdp, "OSDP_ACT_" + n.upper()) for n in R.NAMES}


def rand(*shape, std=1.0, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(hash((shape, seed)) % (1 << 31))
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


class Op:
    """One operator: W in N shards, flat pieces of ceil(I O / N)."""

    def __init__(self, T, I, O, N, k=1, split=osdp.OSDP_SPLIT_OUT_FEATURES, seed=0, zdp=None, staging=osdp.OSDP_STAGING_AUTO):
        self.T, self.I, self.O, self.N, self.k = T, I, O, N, k
        L = -(-I * O // N)
        flat = torch.full((N * L,), float("nan"), dtype=torch.bfloat16, device="cuda")
        flat[:I * O] = rand(I * O, std=I ** -0.5, seed=seed)
        self.W, self.w = flat[:I * O].view(I, O), [s.clone() for s in flat.split(L)]
        self.X = rand(T, I, seed=seed + 1)
        self.plan = osdp.Plan([k], staging=staging, split_dim_per_op=[split], zdp_mask=None if zdp is None else [zdp])
        self.ws = None

    def workspace(self, bwd):
        need, _ = osdp.osdp_split_linear_epilogue_workspace_bytes(self.T, self.I, self.O, self.N, self.k, bwd, plan=self.plan)
        self.ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN, whatever is read of it first)
        return self.ws

    def fwd(self, Y, stream=None, copy=None, **epilogue):
        osdp.osdp_split_linear_fwd_epilogue(self.X, self.w, Y, self.k, self.workspace(False), epilogue=osdp.Epilogue(**epilogue), plan=self.plan,
                                            stream_compute=stream, stream_copy=copy)
        return Y

    def bwd(self, dY, stream=None, **epilogue):
        dX = torch.full((self.T, self.I), float("nan"), dtype=torch.bfloat16, device="cuda")
        dW = [torch.full_like(s, float("nan")) for s in self.w]
        osdp.osdp_split_linear_bwd_epilogue(self.X, dY, self.w, dX, dW, self.k, self.workspace(True), epilogue=osdp.EpilogueGrad(**epilogue),
                                            plan=self.plan, stream_compute=stream)
        return dX, torch.cat(dW)[:self.I * self.O]

    def z(self, bias):
        z = self.X.double() @ self.W.double()
        return z if bias is None else z + bias.double()

    def out(self, fill=float("nan"), pad=0):
        return torch.full((self.T, self.O + pad), fill, dtype=torch.bfloat16, device="cuda")[:, pad // 2:pad // 2 + self.O]


def close(got, want, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got - want).abs() - bound
    assert off.max().item() <= 0, f"{what}: {int((off > 0).sum())} values beyond the bound, by up to {off.max().item():.3e}"


def check_forward(op, act, bias=None, residual=None, Y=None, Z=None):
    z = op.z(bias)
    rms = z.square().mean().sqrt() if z.numel() else 0.0
    a = R.act(act, z)
    y = a if residual is None else a + residual.double()
    if Y is not None:
        close(Y, y, 2.0 ** -8 * y.abs() + 2.0 ** -15 * a.abs() + 1.13e-3 * rms, "Y")
    if Z is not None:
        close(Z, z, 2.0 ** -8 * z.abs() + 1e-3 * rms, "Z")


# (T, I, O, N, k): few tokens, tiles of every kind, shards that are no row blocks, sizes that nothing divides but 8
SHAPES = [(1, 64, 8, 1, 1), (1, 4096, 16384, 8, 1), (3, 200, 136, 17, 1), (16, 256, 32768, 4, 1), (33, 1024, 520, 8, 1), (64, 2056, 264, 3, 1), (65, 512, 8448, 8, 1),
          (128, 256, 1024, 2, 4), (129, 256, 1024, 2, 4), (255, 1000, 72, 1, 1), (500, 2560, 2560, 8, 2), (513, 320, 640, 5, 2), (777, 1504, 3200, 4, 2),
          (1024, 520, 2056, 40, 1), (1500, 4096, 4096, 8, 4), (2049, 128, 1032, 2, 1), (3001, 1024, 3200, 8, 1), (4096, 2560, 10240, 8, 4), (8192, 1024, 4096, 8, 4),
          # one shard, and shards of a multiple of 8 rows, which dX's tiles end with
          (700, 1112, 1608, 1, 3), (200, 2616, 352, 1, 2), (130, 72, 136, 1, 1), (600, 1664, 512, 8, 4), (2000, 1088, 2048, 4, 2), (150, 128, 2048, 16, 1), (400, 640, 9000, 8, 3),
          # products that run in parts of a long reduction where they are staged, and one that does not
          (600, 16384, 264, 3, 1), (300, 24576, 528, 3, 3), (600, 16384, 264, 8, 1), (2, 31824, 1672, 1, 1), (33, 16384, 512, 8, 1),
          (128, 9992, 136, 17, 1), (215, 920, 20288, 16, 8), (193, 16080, 544, 32, 4), (337, 19336, 352, 11, 4), (1488, 672, 984, 9, 1), (900, 712, 952, 7, 1), (7, 23080, 744, 2, 1), (200, 6200, 664, 8, 1), (130, 8192, 8, 8, 1), (90, 8192, 16384, 8, 2)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("act", R.NAMES)
def test_forward(shape, act):
    op = Op(*shape)
    bias = rand(op.O, std=0.5, seed=7, dtype=torch.float32 if act in ("gelu", "none") else torch.bfloat16)
    residual = rand(op.T, op.O, seed=8)
    Y, Z = op.out(), op.out()
    op.fwd(Y, bias=bias, activation=ACTS[act], residual=residual, z=Z)
    check_forward(op, act, bias, residual, Y, Z)


@pytest.mark.parametrize("shape", [(7, 256, 512, 2, 1), (300, 512, 768, 8, 2), (2000, 512, 1280, 8, 1)], ids=str)
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("with_z", [False, True])
def test_each_part_can_be_left_out(shape, with_bias, with_residual, with_z):
    op = Op(*shape)
    bias = rand(op.O, std=0.5, seed=3) if with_bias else None
    residual = rand(op.T, op.O, seed=4) if with_residual else None
    Y, Z = op.out(), op.out() if with_z else None
    op.fwd(Y, bias=bias, activation=ACTS["silu"], residual=residual, z=Z)
    check_forward(op, "silu", bias, residual, Y, Z)


@pytest.mark.parametrize("T", [5, 400, 1300])
def test_nothing_but_the_product_is_the_product_bit_by_bit(T):
    """Without anything, and with a bias and residual of zeros (adding which changes no bit but the sign of zero)."""
    op = Op(T, 512, 1024, 8, 2)
    plain = op.out()
    osdp.osdp_split_linear_fwd(op.X, op.w, plain, op.k, op.workspace(False), plan=op.plan)
    assert torch.equal(op.fwd(op.out()).view(torch.int16), plain.view(torch.int16))
    assert torch.equal(op.fwd(op.out(), bias=torch.zeros(op.O, device="cuda"), residual=torch.zeros_like(plain)), plain)


@pytest.mark.parametrize("T,I,O", [(40, 512, 1024), (300, 512, 1024), (1300, 512, 1024), (4096, 1024, 2048), (20, 8192, 512), (100, 8192, 512), (300, 4096, 512), (700, 8192, 512)])
def test_cuts_modes_and_shards_change_no_bit(T, I, O):
    bias, residual = rand(O, seed=1), rand(T, O, seed=2)
    how = dict(bias=bias, activation=ACTS["gelu"], residual=residual)
    cut = {(512, 1024): 18, (1024, 2048): 13, (8192, 512): 26, (4096, 512): 13}[I, O]
    # shards that are blocks of a multiple of 64 rows, or one; shards that are not may have another order of sums from 129 tokens on
    blocks = [(8, 1, 0, 1), (1, 1, 0, 1), (8, 4, 0, 1), (8, 4, 0, 2), (8, 4, 0, 3), (8, 4, 1, 1), (8, 2, 1, 2), (8, 4, 3, 1), (4, 2, 0, 1), (1, 4, 0, 1), (1, 2, 1, 2)]
    flat = [(cut, 1, 0, 1), (cut, 4, 0, 1), (cut, 2, 0, 2), (cut, 1, 1, 1)]
    if T <= 128 or not in_parts(T, I, O):  # (row slices that are staged go on in one chain, not in parts)
        flat.append((cut, 4, 1, 1))
    for plans in ([blocks + flat] if T <= 128 else [blocks, flat]):
        want = None
        for N, k, split, staging in plans:
            op = Op(T, I, O, N, k, split, staging=staging)
            got = op.fwd(op.out(), **how)
            check_forward(op, "gelu", bias, residual, got)
            assert want is None or torch.equal(got, want), (N, k, split, staging)
            want = got


@pytest.mark.parametrize("switch,values", [("tile", range(4)), ("gemm_generic", (1,)), ("persistent", (0, 1)), ("four_wave", (0, 1)), ("small_tile", (0, 1)), ("deep", (0,)),
                                           ("split_launch", (0,)), ("fused_gather", (0, 1)), ("fwd_pair", (0, 1)), ("poison_staging", (1,)), ("recut", (0, 1))])
def test_every_kernel_gives_the_same_bits(switch, values):
    """Every tile and schedule that can run a forward launch, over shards that are row blocks and over such that are not."""
    bias, how = rand(1600, seed=1), {}
    for T, N in ((600, 8), (1111, 8), (4000, 5)):
        for k, split, staging in ((4, 0, 2), (2, 1, 2), (1, 0, 1)):
            op = Op(T, 1024, 1600, N, k, split, staging=staging)
            how = dict(bias=bias, activation=ACTS["gelu_tanh"], residual=rand(T, 1600, seed=2), z=op.out())
            want, want_z = op.fwd(op.out(), **how), how["z"].clone()
            check_forward(op, "gelu_tanh", bias, how["residual"], want, want_z)
            for v in values:
                osdp.osdp_debug_option(switch, v)
                try:
                    how["z"] = op.out()
                    got = op.fwd(op.out(), **how)
                    torch.cuda.synchronize()
                finally:
                    osdp.osdp_debug_option(switch, 0 if switch in ("gemm_generic", "poison_staging") else -1)
                assert torch.equal(got, want) and torch.equal(how["z"], want_z), (switch, v, T, N, k, split)


@pytest.mark.parametrize("T,I,O", [(20, 512, 1024), (200, 512, 1024), (900, 512, 1024), (20, 4096, 512), (300, 4096, 512), (300, 512, 8192)])
@pytest.mark.parametrize("split", [osdp.OSDP_SPLIT_OUT_FEATURES, osdp.OSDP_SPLIT_IN_FEATURES])
def test_slices_in_dp_mode(T, I, O, split):
    """Slices 0 and 2 of 4 replicated, the shards' part of them poisoned: the bits of the plan that gathers all, but where slices that the
    sum goes over are a chain and the whole runs in parts."""
    op, mixed = Op(T, I, O, 8, 4, split), Op(T, I, O, 8, 4, split, zdp=0b1010)
    bias, residual = rand(O, seed=1), rand(T, O, seed=2)
    dY, Z = rand(T, O, seed=3), rand(T, O, seed=4)
    full, step = mixed.W.contiguous(), (I if split else O) // 4
    replicas = [full[j * step:(j + 1) * step] if split else full[:, j * step:(j + 1) * step] for j in range(4)]
    w_dp = [replicas[j] if j in (0, 2) else None for j in range(4)]
    dw = torch.full_like(full, float("nan"))
    dw_dp = [(dw[j * step:(j + 1) * step] if split else dw[:, j * step:(j + 1) * step]) if j in (0, 2) else None for j in range(4)]
    how = dict(bias=bias, activation=ACTS["relu"], residual=residual)
    want = op.fwd(op.out(), **how)
    got = mixed.out()
    osdp.osdp_split_linear_fwd_epilogue(mixed.X, mixed.w, got, 4, mixed.workspace(False), epilogue=osdp.Epilogue(**how), plan=mixed.plan, w_dp=w_dp,
                                        ld_dp=O)
    check_forward(mixed, "relu", bias, residual, got)
    assert T > 128 and split and in_parts(T, I, O) or torch.equal(got, want)
    dz, dz2, db, db2 = op.out(), op.out(), torch.zeros(O, device="cuda"), torch.ones(O, device="cuda")
    dX, dW = op.bwd(dY, activation=ACTS["relu"], z=Z, dz=dz, dbias=db)
    dX2 = torch.full_like(dX, float("nan"))
    dws = [torch.full_like(s, float("nan")) for s in mixed.w]
    osdp.osdp_split_linear_bwd_epilogue(mixed.X, dY, mixed.w, dX2, dws, 4, mixed.workspace(True), plan=mixed.plan, w_dp=w_dp, ld_dp=O, dw_dp=dw_dp,
                                        epilogue=osdp.EpilogueGrad(activation=ACTS["relu"], z=Z, dz=dz2, dbias=db2))
    assert torch.equal(dz2, dz) and torch.equal(db2, db)
    flat = torch.cat(dws).view(I, O)
    flat = torch.where(torch.isnan(flat), dw, flat)
    check_products(mixed, dz, dX2, flat.flatten())
    assert torch.equal(flat, dW.view(I, O))
    assert T > 128 and not split and in_parts(T, O, I) or torch.equal(dX2, dX)


@pytest.mark.parametrize("T", [9, 600])
def test_places_in_wider_matrices_and_a_residual_in_place(T):
    """Y, Z and the residual as parts of one wide matrix; what lies beside them stays as it was."""
    op = Op(T, 256, 520, 2)
    bias = rand(520, seed=1)
    wide = rand(T, 4 * 528, seed=2)
    before = wide.clone()
    Y, Z, residual = wide[:, :520], wide[:, 528:1048], wide[:, 1056:1576]
    op.fwd(Y, bias=bias, activation=ACTS["gelu"], residual=residual, z=Z)
    check_forward(op, "gelu", bias, before[:, 1056:1576], Y, Z)
    changed = (wide.view(torch.int16) != before.view(torch.int16)).any(0).nonzero().view(-1).tolist()
    assert all(c < 520 or 528 <= c < 1048 for c in changed)
    r = rand(T, 520, seed=5)
    Y = r.clone()
    op.fwd(Y, bias=bias, activation=ACTS["silu"], residual=Y)
    assert torch.equal(Y, op.fwd(op.out(), bias=bias, activation=ACTS["silu"], residual=r))


def test_no_tokens():
    op = Op(0, 64, 128, 2)
    op.fwd(op.out(), bias=rand(128), activation=ACTS["gelu"])
    for dtype in (torch.float32, torch.bfloat16):
        db = torch.full((128,), float("nan"), dtype=dtype, device="cuda")
        _, dW = op.bwd(op.out(), activation=ACTS["gelu"], z=op.out(), dz=op.out(), dbias=db)
        assert (db == 0).all() and (dW == 0).all()


def through(op, act, values, dtype=torch.float32):
    """Y where X . W is 0 and the bias runs through `values`: what the activation makes of fp32 numbers."""
    op.X.zero_()
    Y, Z = op.out(), op.out()
    op.fwd(Y, bias=values.to(dtype), activation=ACTS[act], z=Z)
    return Y, Z


@pytest.mark.parametrize("act", R.NAMES)
@pytest.mark.parametrize("T", [1, 600])
def test_the_whole_range_of_activations(act, T):
    """Values from 2^-100 to 2^100 of both signs, and steps through -12 .. 12: off by 2^-8 for bf16 and 2^-15 for the fp32 arithmetic."""
    e = torch.exp2(torch.linspace(-100, 100, 1601, dtype=torch.float64))
    v = torch.cat([-e, e, torch.linspace(-12, 12, 4894, dtype=torch.float64)]).float().cuda()
    op = Op(T, 64, v.numel(), 1)
    Y, _ = through(op, act, v)
    want = R.act(act, v.double())
    # (below 2^-126 the hardware's exponential gives 0)
    close(Y[0], want, (2.0 ** -8 + 2.0 ** -15) * want.abs() + 1e-36, "Y")
    assert torch.equal(Y, Y[:1].expand(T, -1))


@pytest.mark.parametrize("T", [2, 600])
def test_infinities_and_nan(T):
    inf, nan = float("inf"), float("nan")
    v = torch.tensor([inf, -inf, nan, 0.0, -0.0, 3.0, -3.0, 1.0]).cuda()
    op = Op(T, 64, 8, 1)
    for act in R.NAMES:
        Y, Z = through(op, act, v)
        low = {"none": -inf, "relu": 0.0}.get(act, nan)
        want = torch.tensor([inf, low, nan]).cuda()
        assert torch.equal(torch.nan_to_num(Y[0, :3].float(), 7.0), torch.nan_to_num(want, 7.0)), act
        assert torch.isnan(Z[:, 2]).all() and torch.isfinite(Y[:, 3:]).all() and (Y[:, 3:5] == 0).all()


def in_parts(M, K, N):
    """Whether a product of few 128 x 128 tiles runs in parts of its reduction, each summed up by itself."""
    tiles = -(-M // 128) * -(-N // 128)
    parts = min(256 // tiles, K // 512, 32)
    return parts >= 2 and K - K // parts >= 1500


def check_products(op, dz, dX, dW):
    for got, want, what in ((dX, dz.double() @ op.W.double().t().contiguous(), "dX"), (dW.view(op.I, op.O), op.X.double().t().contiguous() @ dz.double(), "dW")):
        close(got, want, 2.0 ** -8 * want.abs() + 1e-3 * want.square().mean().sqrt(), what)


# ---- backward ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("act", R.NAMES)
def test_backward(shape, act):
    op = Op(*shape)
    dtype = torch.float32 if act in ("gelu", "none") else torch.bfloat16
    dY, Z = rand(op.T, op.O, seed=5), rand(op.T, op.O, std=1.5, seed=6)
    db, dz = torch.full((op.O,), float("nan"), dtype=dtype, device="cuda"), op.out() if act != "none" else None
    dX, dW = op.bwd(dY, activation=ACTS[act], z=None if dz is None else Z, dz=dz, dbias=db)
    want = dY.double() * R.slope(act, Z.double())
    if dz is not None:
        close(dz, want, (2.0 ** -8 + 2.0 ** -23) * want.abs() + 2.0 ** -15 * dY.double().abs(), "dZ")
    s = want.sum(0)
    terms = (2.0 ** -15 * dY.double().abs()).sum(0) + (op.T + 2) * 2.0 ** -24 * want.abs().sum(0)
    close(db, s, terms + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * (s.abs() + terms), "db")
    ref = Op(*shape)
    rX, rW = torch.full_like(dX, float("nan")), [torch.full_like(w, float("nan")) for w in ref.w]
    osdp.osdp_split_linear_bwd(ref.X, dY if dz is None else dz, ref.w, rX, rW, ref.k, ref.workspace(True), plan=ref.plan)
    check_products(op, dY if dz is None else dz, dX, dW)
    T, I, O = op.T, op.I, op.O
    if not (in_parts(T, O, I) or T <= 128 and O > 1000):
        assert torch.equal(dX, rX)
    if not in_parts(I, T, O):
        assert torch.equal(dW, torch.cat(rW)[:op.I * op.O])


@pytest.mark.parametrize("T,I,O", [(2, 272, 14464), (100, 64, 8192), (300, 256, 8192), (8192, 512, 512), (4100, 544, 544), (3000, 128, 64), (5000, 64, 8192)])
@pytest.mark.parametrize("place", ["apart", "dX for X"])
def test_products_of_few_tiles(T, I, O, place):
    """Those that run in parts, whatever the cut and the shards, and dX in the place of X."""
    dY, Z = rand(T, O, seed=5), rand(T, O, seed=6)
    first = None
    for N, k, split in [(1, 1, 0), (8, 4, 0), (8, 2, 1), (4, 2, 3)]:
        op = Op(T, I, O, N, k, split)
        X, dz, dW = op.X.clone(), op.out(), [torch.full_like(s, float("nan")) for s in op.w]
        dX = op.X if place == "dX for X" else torch.full_like(X, float("nan"))
        osdp.osdp_split_linear_bwd_epilogue(op.X, dY, op.w, dX, dW, k, op.workspace(True), plan=op.plan,
                                            epilogue=osdp.EpilogueGrad(activation=ACTS["silu"], z=Z, dz=dz, dbias=torch.empty(O, device="cuda")))
        op.X = X
        dW = torch.cat(dW)[:I * O]
        check_products(op, dz, dX, dW)
        assert first is None or torch.equal(dW, first)
        first = dW


def test_the_gradients_are_the_differences_of_the_forward_pass():
    """sum(Y dY) along random directions of X, W, b and R, by central differences of the formula in 64 bits, against the kernels'
    gradients: each is off by its own bound, 2^-7 of it (two roundings, dZ's and its own) and 2e-3 of the root mean square."""
    op = Op(300, 256, 512, 4, 2)
    bias, residual, dY = rand(512, seed=1, dtype=torch.float32), rand(300, 512, seed=2), rand(300, 512, seed=3)
    for act in R.NAMES[2:]:
        Z, dz, db = op.out(), op.out(), torch.empty_like(bias)
        op.fwd(op.out(), bias=bias, activation=ACTS[act], residual=residual, z=Z)
        dX, dW = op.bwd(dY, activation=ACTS[act], z=Z, dz=dz, dbias=db)
        x, w, b, dy, h = op.X.double(), op.W.double(), bias.double(), dY.double(), 1e-5
        for grad, at in ((dX.double(), 0), (dW.double().view(256, 512), 1), (db.double(), 2)):
            u = torch.randn(grad.shape, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(at))
            def loss(s):
                p = [x, w, b]
                p[at] = p[at] + s * h * u
                return (R.act(act, p[0] @ p[1] + p[2]) * dy).sum().item()
            by_difference, by_kernel = (loss(1) - loss(-1)) / (2 * h), (grad * u).sum().item()
            # (Z is rounded to 2^-8 of it before its slope is taken: independent errors, as those of the roundings are)
            bound = 6 * ((2.0 ** -7 * grad.abs() * u.abs()).square().sum().sqrt() + 2e-2 * grad.square().mean().sqrt() * u.norm()).item()
            assert abs(by_difference - by_kernel) <= bound, (act, at, by_difference, by_kernel, bound)


@pytest.mark.parametrize("T", [1, 100, 300, 3000])
def test_dz_in_place_and_no_gradient_of_the_bias(T):
    op = Op(T, 256, 392, 2)
    dY, Z = rand(T, 392, seed=5), rand(T, 392, seed=6)
    want = op.out()
    db = torch.empty(392, device="cuda")
    dX, dW = op.bwd(dY, activation=ACTS["gelu"], z=Z, dz=want, dbias=db)
    for at in ("dY", "Z"):
        dy, z = dY.clone(), Z.clone()
        dz = dy if at == "dY" else z
        db2 = torch.empty_like(db) if at == "Z" else None
        dX2, dW2 = op.bwd(dy, activation=ACTS["gelu"], z=z, dz=dz, dbias=db2)
        assert torch.equal(dz, want) and torch.equal(dX2, dX) and torch.equal(dW2, dW) and (db2 is None or torch.equal(db2, db))


@pytest.mark.parametrize("act", R.NAMES[1:])
def test_slopes_over_the_whole_range(act):
    e = torch.exp2(torch.linspace(-100, 100, 2001))
    z = torch.cat([-e, e, torch.linspace(-12, 12, 4006)]).bfloat16().cuda().view(1, -1)
    op = Op(1, 64, z.numel(), 1)
    dz = op.out()
    op.bwd(torch.ones_like(z), activation=ACTS[act], z=z, dz=dz)
    want = R.slope(act, z.double())
    want = torch.where(torch.isfinite(want), want, (z > 0).double())  # (the cube of 2^100 leaves the range even of 64 bits)
    close(dz, want, 2.0 ** -8 * want.abs() + 2.0 ** -15, act)


def test_offsets_beyond_32_bits():
    """Rows 2^19 elements apart, 8 GB of residual, Z, dY: the last rows lie beyond 2^31 elements and 2^32 bytes."""
    T, ld = 4200, 1 << 19
    op = Op(T, 64, 72, 1)
    wide = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)
    Y, Z, residual, dY, dz = (wide[:, 128 * i:128 * i + 72] for i in range(5))
    residual.copy_(rand(T, 72, seed=1))
    dY.copy_(rand(T, 72, seed=2))
    bias, db = rand(72, seed=3), torch.empty(72, dtype=torch.bfloat16, device="cuda")
    op.fwd(Y, bias=bias, activation=ACTS["silu"], residual=residual, z=Z)
    check_forward(op, "silu", bias, residual, Y, Z)
    dX, dW = op.bwd(dY, activation=ACTS["silu"], z=Z, dz=dz, dbias=db)
    near = Op(T, 64, 72, 1)
    dz2, db2 = near.out(), torch.empty_like(db)
    dX2, dW2 = near.bwd(dY.contiguous(), activation=ACTS["silu"], z=Z.contiguous(), dz=dz2, dbias=db2)
    assert torch.equal(dz, dz2) and torch.equal(dX, dX2) and torch.equal(dW, dW2) and torch.equal(db, db2)


# (in one launch and staged; then what runs in parts: few tokens, tiles forward, tiles backward, few-token kernel for more of them)
@pytest.mark.parametrize("T,I,O,N", [(4, 256, 512, 8), (700, 256, 512, 8), (33, 4096, 512, 8), (300, 4096, 512, 8), (4100, 512, 512, 8), (200, 1024, 1024, 32)])
def test_a_captured_graph_replays_on_other_inputs(T, I, O, N):
    """Forward and backward captured once, replayed with new inputs in the same place, eager work in between."""
    op = Op(T, I, O, N, 2)
    bias, residual, dY = rand(O, seed=1), rand(T, O, seed=2), rand(T, O, seed=3)
    Y, Z, dz, db = op.out(), op.out(), op.out(), torch.empty_like(bias)
    dX, dW = torch.empty_like(op.X), [torch.empty_like(s) for s in op.w]
    wf, wb = op.workspace(False), op.workspace(True)

    def run(stream):
        osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, Y, 2, wf, plan=op.plan, stream_compute=stream,
                                            epilogue=osdp.Epilogue(bias=bias, activation=ACTS["gelu"], residual=residual, z=Z))
        osdp.osdp_split_linear_bwd_epilogue(op.X, dY, op.w, dX, dW, 2, wb, plan=op.plan, stream_compute=stream,
                                            epilogue=osdp.EpilogueGrad(activation=ACTS["gelu"], z=Z, dz=dz, dbias=db))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    run(stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(stream)
    for seed in range(4):
        op.X.copy_(rand(T, I, seed=50 + seed))
        dY.copy_(rand(T, O, seed=60 + seed))
        outs = [Y, Z, dz, db, dX, *dW]
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        run(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), seed


@pytest.mark.parametrize("T,I", [(700, 512), (40, 8192), (300, 8192)])
def test_two_streams_with_workspaces_of_their_own(T, I):
    ops = [Op(T, I, 1024, 8, 2, seed=s) for s in (0, 10)]
    bias = rand(1024, seed=1)
    want = [op.fwd(op.out(), bias=bias, activation=ACTS["gelu"]) for op in ops]
    streams, got, spaces = [torch.cuda.Stream() for _ in ops], [op.out() for op in ops], [op.workspace(False) for op in ops]
    torch.cuda.synchronize()
    for _ in range(5):
        for op, y, s, ws in zip(ops, got, streams, spaces):
            osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, y, op.k, ws, plan=op.plan, stream_compute=s,
                                                epilogue=osdp.Epilogue(bias=bias, activation=ACTS["gelu"]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_binding_refuses_what_does_not_fit():
    op = Op(16, 64, 128, 2)
    Y, bias = op.out(), rand(128)
    wrong = [dict(bias=rand(120)), dict(bias=rand(128).half()), dict(bias=rand(256)[::2]), dict(bias=rand(128).cpu()), dict(residual=rand(16, 120)),
             dict(residual=rand(16, 128).float()), dict(residual=rand(128, 16).t()), dict(residual=rand(1, 128).expand(16, 128)), dict(z=Y), dict(z=op.X.repeat(1, 2).cpu()),
             dict(bias=bias, activation=17)]
    for w in wrong:
        with pytest.raises(osdp.OsdpError):
            op.fwd(Y, **w)
    for X, y, shards in ((op.X.float(), Y, op.w), (op.X, Y.float(), op.w), (op.X, Y[:8], op.w), (op.X, Y, [s.float() for s in op.w]), (op.X, Y, [s[:-8] for s in op.w])):
        with pytest.raises(osdp.OsdpError):
            osdp.osdp_split_linear_fwd_epilogue(X, shards, y, 1, op.workspace(False), epilogue=osdp.Epilogue(bias=bias))
    dw = [torch.empty_like(s) for s in op.w]
    for kind in (dw[:1], [d.float() for d in dw], [d[:-8] for d in dw]):
        with pytest.raises(osdp.OsdpError):
            osdp.osdp_split_linear_bwd_epilogue(op.X, Y, op.w, torch.empty_like(op.X), kind, 1, op.workspace(True), epilogue=osdp.EpilogueGrad(dbias=bias))
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, Y, 1, torch.empty(0, dtype=torch.uint8, device="cuda"), epilogue=osdp.Epilogue(bias=bias))


def test_a_transformer_layer_runs_together():
    """qkv with bias, norms and rotation in place, proj onto the residual stream, up with gelu, down onto the residual stream; then all of
    it backward.  Each step is checked against its formula in 64 bits on the very tensors that the step before it left."""
    T, h, f, D = 700, 512, 1024, 64
    n_heads = h // D
    qkv, proj, up, down = Op(T, h, 3 * h, 8, 2, seed=1), Op(T, h, h, 8, seed=2), Op(T, h, f, 8, 2, seed=3), Op(T, f, h, 8, 2, seed=4)
    bias = [rand(o, std=0.2, seed=9) for o in (3 * h, h, f, h)]
    x0 = qkv.X
    rows = qkv.fwd(qkv.out(), bias=bias[0])
    check_forward(qkv, "none", bias[0], Y=rows)
    pos, freqs = torch.arange(T, device="cuda"), 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") * 2 / D)
    g = [rand(D, std=0.1, seed=11 + i, dtype=torch.float32).add_(1).bfloat16() for i in range(2)]
    q, k = rows[:, :h].unflatten(1, (n_heads, D)), rows[:, h:2 * h].unflatten(1, (n_heads, D))
    kept = rows.clone()  # (what the pass back needs)
    kq, kk = kept[:, :h].unflatten(1, (n_heads, D)), kept[:, h:2 * h].unflatten(1, (n_heads, D))
    how = dict(positions=pos, freqs=freqs, q_weight=g[0], k_weight=g[1])
    osdp.osdp_qk_norm_rope_fwd(q, k, q, k, **how)
    for got, x, w in ((q, kq, g[0]), (k, kk, g[1])):
        want = R.qk(x.double(), pos, freqs, w, 1e-6, True, False)
        close(got, want, 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True), "heads")
    assert torch.equal(rows[:, 2 * h:], kept[:, 2 * h:])
    proj.X = rows[:, 2 * h:]  # (in the place of attention: the values)
    x1 = proj.fwd(proj.out(), bias=bias[1], residual=x0)
    check_forward(proj, "none", bias[1], x0, x1)
    up.X = x1
    Z = up.out()
    down.X = up.fwd(up.out(), bias=bias[2], activation=ACTS["gelu"], z=Z)
    check_forward(up, "gelu", bias[2], None, down.X, Z)
    x2 = down.fwd(down.out(), bias=bias[3], residual=x1)
    check_forward(down, "none", bias[3], x1, x2)

    dY = rand(T, h, seed=20)
    db = [torch.empty_like(b) for b in bias]

    def products(op, dz, dX, dW):
        # (2^-8 of what is rounded, 1e-3 of the root mean square for the sums: as for the products' other tests)
        for got, want, what in ((dX, dz.double() @ op.W.double().t().contiguous(), "dX"), (dW.view(op.I, op.O), op.X.double().t().contiguous() @ dz.double(), "dW")):
            close(got, want, 2.0 ** -8 * want.abs() + 1e-3 * want.square().mean().sqrt(), what)

    d_act, dW = down.bwd(dY, dbias=db[3])
    products(down, dY, d_act, dW)
    dz = up.out()
    d1, dW = up.bwd(d_act, activation=ACTS["gelu"], z=Z, dz=dz, dbias=db[2])
    want = d_act.double() * R.slope("gelu", Z.double())
    close(dz, want, (2.0 ** -8 + 2.0 ** -23) * want.abs() + 2.0 ** -15 * d_act.double().abs(), "dZ")
    products(up, dz, d1, dW)
    d1 = d1 + dY
    dv, dW = proj.bwd(d1, dbias=db[1])
    products(proj, d1, dv, dW)
    d_rows = qkv.out()
    d_rows[:, 2 * h:] = dv
    dq_out, dk_out = rand(T, n_heads, D, seed=30), rand(T, n_heads, D, seed=31)  # (what attention would send back)
    dg = [torch.empty_like(w) for w in g]
    ws = torch.empty(osdp.osdp_qk_norm_rope_bwd_workspace_bytes(T, n_heads, n_heads, D), dtype=torch.uint8, device="cuda")
    dq, dk = d_rows[:, :h].unflatten(1, (n_heads, D)), d_rows[:, h:2 * h].unflatten(1, (n_heads, D))
    osdp.osdp_qk_norm_rope_bwd(kq, kk, dq_out, dk_out, dq, dk, dg[0], dg[1], ws, **how)
    for got, gw, x, dy, w in ((dq, dg[0], kq, dq_out, g[0]), (dk, dg[1], kk, dk_out, g[1])):
        dx, dw = R.qk_back(x.double(), dy.double(), pos, freqs, w, 1e-6, True, False)
        close(got, dx, 2.0 ** -8 * dx.abs() + 2.0 ** -16 * dx.abs().amax(-1, keepdim=True), "d heads")
        close(gw, dw, 2.0 ** -8 * dw.abs() + 1e-4 * dw.square().mean().sqrt(), "d weight")
    dx, dW = qkv.bwd(d_rows, dbias=db[0])
    products(qkv, d_rows, dx, dW)
    s = d_rows.double().sum(0)
    close(db[0], s, 2.0 ** -8 * s.abs() + T * 2.0 ** -24 * d_rows.double().abs().sum(0), "db")


@pytest.mark.parametrize("T", [65, 100, 128])
def test_wide_operators_of_a_hundred_tokens(T):
    """More than 8192 output columns over shards of a multiple of 64 rows: from 65 tokens on the tiles' kernels, in parts of the
    reduction.  All plans give the same bits but one with row slices in DP mode, which go on in one chain."""
    I, O = 4096, 8448
    assert in_parts(T, I, O)
    bias, residual = rand(O, seed=1), rand(T, O, seed=2)
    how = dict(bias=bias, activation=ACTS["gelu"], residual=residual)
    want = None
    for N, k, split, staging, zdp in [(8, 1, 0, 1, None), (1, 1, 0, 1, None), (8, 4, 0, 1, None), (8, 4, 0, 2, None), (8, 4, 1, 1, None), (8, 2, 1, 2, None), (64, 4, 1, 3, None),
                                      (8, 4, 0, 1, 0b1010), (8, 4, 1, 1, 0b1010)]:
        op = Op(T, I, O, N, k, split, staging=staging, zdp=zdp)
        if zdp is None:
            got = op.fwd(op.out(), **how)
        else:
            w, step, got = op.W.contiguous(), (I if split else O) // k, op.out()
            w_dp = [w[j * step:(j + 1) * step] if split else w[:, j * step:(j + 1) * step] for j in range(k)]
            osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, got, k, op.workspace(False), epilogue=osdp.Epilogue(**how), plan=op.plan, w_dp=w_dp, ld_dp=O)
        if zdp is None or not split:
            assert want is None or torch.equal(got, want), (N, k, split, staging, zdp)
            want = got
        check_forward(op, "gelu", bias, residual, got)


@pytest.mark.parametrize("T,I,O,k", [(300, 520, 4168, 5), (300, 520, 4160, 5), (4168, 264, 520, 3), (100, 8448, 4096, 4), (40, 512, 4096, 4)])
def test_gradients_of_products_in_parts_are_the_same_for_every_plan(T, I, O, k):
    """Whatever the shards, cuts and modes of the slices, but that dX of column slices in DP mode goes on in one chain, and that of 65 to
    128 tokens and more than 8192 in-features is the few-token kernel's, or the tiles' where shards are a multiple of 64 rows."""
    dY, Z, want, want_dX = rand(T, O, seed=3), rand(T, O, seed=4), None, {}
    for N, k_, split, staging, zdp in [(1, 1, 0, 1, None), (8, 1, 0, 1, None), (1, k, 1, 1, None), (8, k, 1, 1, None), (8, k, 1, 2, None), (8, k, 0, 1, None), (8, k, 0, 2, None), (8, k, 1, 1, 0b11010),
                                      (8, k, 0, 1, 0b11010)]:
        if split == 0 and O % (8 * k_):
            continue
        op = Op(T, I, O, N, k_, split, staging=staging, zdp=zdp)
        full, step = op.W.contiguous(), (I if split else O) // k_
        dw = torch.full_like(full, float("nan"))
        cut = lambda m: [m[j * step:(j + 1) * step] if split else m[:, j * step:(j + 1) * step] for j in range(k_)]  # noqa: E731
        dz, dX, dws = op.out(), torch.full_like(op.X, float("nan")), [torch.full_like(s, float("nan")) for s in op.w]
        osdp.osdp_split_linear_bwd_epilogue(op.X, dY, op.w, dX, dws, k_, op.workspace(True), plan=op.plan, epilogue=osdp.EpilogueGrad(activation=ACTS["gelu"], z=Z, dz=dz),
                                            **({} if zdp is None else dict(w_dp=cut(full), ld_dp=O, dw_dp=cut(dw))))
        dW = torch.cat(dws)[:I * O].view(I, O)
        dW = torch.where(torch.isnan(dW), dw, dW)
        check_products(op, dz, dX, dW.flatten())
        want = dW if want is None else want
        assert torch.equal(dW, want), (N, k_, split, zdp)
        if zdp is None or split:
            kernel = 64 < T <= 128 and I > 8192 and I % (64 * N) == 0
            assert torch.equal(dX, want_dX.setdefault(kernel, dX)), (N, k_, split, zdp)


def test_the_profile_sees_the_pass_for_dz():
    """A backward pass whose dZ (2.1 GB read and written) takes longer than its products: in the span of the profile, and no idle time of it."""
    T, I, O = 32768, 64, 10752
    op, dY, Z = Op(T, I, O, 1), rand(T, O, seed=1), rand(T, O, seed=2)
    dz, dX, dW, ws = torch.empty_like(dY), torch.empty_like(op.X), [torch.empty_like(s) for s in op.w], op.workspace(True)

    def call():
        osdp.osdp_split_linear_bwd_epilogue(op.X, dY, op.w, dX, dW, 1, ws, plan=op.plan, epilogue=osdp.EpilogueGrad(activation=ACTS["relu"], z=Z, dz=dz))

    call()
    torch.cuda.synchronize()
    osdp.osdp_profile_begin(1000)
    for _ in range(4):
        call()
    stats = osdp.osdp_profile_end()
    lay = osdp.osdp_profile_overlap()
    assert stats["gemm_dw"]["launches"] == 4 and stats["gemm_dx"]["launches"] == 4
    assert lay["idle_ms"] < 0.25 * lay["span_ms"], (lay, stats)


# (reductions whose last part is shorter: a whole number of K blocks, the end of one, and parts alike; shards of 832 and 512 rows are
# read in place, the others staged)
@pytest.mark.parametrize("T,I,O,N", [(300, 4160, 520, 5), (300, 4160, 520, 8), (300, 8200, 520, 8), (300, 4096, 512, 8), (140, 24584, 264, 1)])
def test_parts_of_a_reduction_give_the_same_bits_in_every_kernel(T, I, O, N):
    assert in_parts(T, I, O)
    op, bias, residual = Op(T, I, O, N), rand(O, seed=1), rand(T, O, seed=2)
    want = want_z = None
    for switches in [dict(tile=3), dict(tile=0), dict(tile=1), dict(tile=2), dict(tile=3, deep=0), dict(tile=1, deep=0), dict(tile=2, deep=0), dict(tile=0, persistent=1),
                     dict(tile=0, persistent=0), dict(tile=0, four_wave=0), dict(tile=0, four_wave=1), dict(gemm_generic=1), dict(tile=3, recut=0)]:
        Z = op.out()
        got = switched(switches, lambda: op.fwd(op.out(), bias=bias, activation=ACTS["gelu"], residual=residual, z=Z))
        if want is None:
            want, want_z = got, Z
            check_forward(op, "gelu", bias, residual, got, Z)
        assert torch.equal(got, want) and torch.equal(Z, want_z), switches
    if N == 5 or I == 4096:  # (no switch: over the shards where they lie)
        assert torch.equal(op.fwd(op.out(), bias=bias, activation=ACTS["gelu"], residual=residual), want)


@pytest.mark.parametrize("T,I,O,slices", [(300, 520, 4168, 5), (4168, 264, 520, 3), (3000, 520, 264, 5)])
@pytest.mark.parametrize("N,sliced", [(1, False), (8, False), (8, True)])
def test_parts_of_the_backward_reductions_give_the_same_bits_in_every_kernel(T, I, O, slices, N, sliced):
    """dX over O and dW over T, with a shorter last part."""
    assert in_parts(T, O, I) or in_parts(I, T, O)
    k = slices if sliced else 1
    op, dY, Z = Op(T, I, O, N, k, osdp.OSDP_SPLIT_IN_FEATURES), rand(T, O, seed=3), rand(T, O, seed=4)
    want = None
    for switches in [dict(tile=3), dict(tile=0), dict(tile=1), dict(tile=2), dict(tile=3, deep=0), dict(tile=1, deep=0), dict(tile=2, deep=0), dict(tile=0, persistent=1),
                     dict(tile=0, four_wave=0), dict(tile=0, four_wave=1), dict(gemm_generic=1), dict(small_tile=0), dict(fused_gather=0), dict()]:
        dz = op.out()
        got = switched(switches, lambda: op.bwd(dY, activation=ACTS["silu"], z=Z, dz=dz, dbias=torch.empty(O, device="cuda")))
        if want is None:
            want = got
            check_products(op, dz, *got)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), switches


def switched(switches, call):
    """What the call gives under these switches of the library."""
    try:
        for name, value in switches.items():
            osdp.osdp_debug_option(name, value)
        got = call()
        torch.cuda.synchronize()
        return got
    finally:
        for name in switches:
            osdp.osdp_debug_option(name, 0 if name in ("gemm_generic", "poison_staging") else -1)


# (slices staged in two slots, by launches of their own: the copy stream gathers one while the product of the other runs)
@pytest.mark.parametrize("T,I,O,N", [(600, 1024, 4096, 32), (1111, 2080, 2048, 8), (300, 8224, 1024, 8), (300, 8224, 8192, 8), (4100, 544, 8192, 8)])
@pytest.mark.parametrize("split", [osdp.OSDP_SPLIT_OUT_FEATURES, osdp.OSDP_SPLIT_IN_FEATURES])
@pytest.mark.parametrize("poison", [0, 1])
def test_two_streams_give_the_bits_of_one(T, I, O, N, split, poison):
    k = 4
    op = Op(T, I, O, N, k, split, staging=osdp.OSDP_STAGING_DOUBLE)
    bias, residual, dY = rand(O, seed=1), rand(T, O, seed=2), rand(T, O, seed=3)
    compute, copy = torch.cuda.Stream(), torch.cuda.Stream()

    def step(streams):
        Y, Z, dz, db = op.out(), op.out(), op.out(), torch.full_like(bias, float("nan"))
        dX, dW = torch.full_like(op.X, float("nan")), [torch.full_like(s, float("nan")) for s in op.w]
        ws, ws_back = op.workspace(False), op.workspace(True)
        torch.cuda.synchronize()
        osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, Y, k, ws, plan=op.plan, **streams,
                                            epilogue=osdp.Epilogue(bias=bias, activation=ACTS["silu"], residual=residual, z=Z))
        osdp.osdp_split_linear_bwd_epilogue(op.X, dY, op.w, dX, dW, k, ws_back, plan=op.plan, **streams,
                                            epilogue=osdp.EpilogueGrad(activation=ACTS["silu"], z=Z, dz=dz, dbias=db))
        torch.cuda.synchronize()
        return [Y, Z, dz, db, dX, torch.cat(dW)[:I * O]]

    switches = dict(fused_gather=0, fwd_pair=0, **(dict(poison_staging=1) if poison else {}))
    want = switched(switches, lambda: step({}))
    check_forward(op, "silu", bias, residual, want[0], want[1])
    check_products(op, want[2], want[4], want[5])
    for _ in range(3):
        got = switched(switches, lambda: step(dict(stream_compute=compute.cuda_stream, stream_copy=copy.cuda_stream)))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T,I,O,N", [(20, 520, 1032, 5), (100, 1024, 512, 32), (200, 1064, 520, 5), (700, 264, 2056, 3), (300, 8200, 520, 8)])
@pytest.mark.parametrize("split", [osdp.OSDP_SPLIT_OUT_FEATURES, osdp.OSDP_SPLIT_IN_FEATURES])
@pytest.mark.parametrize("zdp", [0b00000, 0b00011, 0b10001, 0b01110])
def test_modes_of_slices_over_shards_that_are_no_row_blocks(T, I, O, N, split, zdp):
    """All slices replicated, neighbours that lie together in the replica, the first and last alone: outputs and gradients."""
    k = next(k for k in (5, 4, 3, 2, 1) if ((I if split else O) % (8 * k)) == 0)
    op = Op(T, I, O, N, k, split, zdp=zdp & ((1 << k) - 1))
    bias, residual, dY, Z = rand(O, seed=1), rand(T, O, seed=2), rand(T, O, seed=3), op.out()
    full, step = op.W.contiguous(), (I if split else O) // k
    dw = torch.full_like(full, float("nan"))
    cut = lambda m: [(m[j * step:(j + 1) * step] if split else m[:, j * step:(j + 1) * step]) if not zdp >> j & 1 else None for j in range(k)]  # noqa: E731
    Y, dz, dX, db = op.out(), op.out(), torch.full_like(op.X, float("nan")), torch.full((O,), float("nan"), device="cuda")
    osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, Y, k, op.workspace(False), plan=op.plan, w_dp=cut(full), ld_dp=O,
                                        epilogue=osdp.Epilogue(bias=bias, activation=ACTS["gelu"], residual=residual, z=Z))
    check_forward(op, "gelu", bias, residual, Y, Z)
    dws = [torch.full_like(s, float("nan")) for s in op.w]
    osdp.osdp_split_linear_bwd_epilogue(op.X, dY, op.w, dX, dws, k, op.workspace(True), plan=op.plan, w_dp=cut(full), ld_dp=O, dw_dp=cut(dw),
                                        epilogue=osdp.EpilogueGrad(activation=ACTS["gelu"], z=Z, dz=dz, dbias=db))
    dW = torch.cat(dws)[:I * O].view(I, O)
    check_products(op, dz, dX, torch.where(torch.isnan(dW), dw, dW).flatten())


def test_calls_of_two_threads_at_once():
    """Each with tensors, a workspace and a stream of its own: the results of calls one after another."""
    shapes = [(33, 1024, 520, 8, 5), (300, 4096, 512, 8, 4)]
    ops = [Op(*s, seed=10 * i) for i, s in enumerate(shapes)]
    state = []
    for op in ops:
        s = dict(bias=rand(op.O, seed=1), residual=rand(op.T, op.O, seed=2), dY=rand(op.T, op.O, seed=3), stream=torch.cuda.Stream(), ws=op.workspace(False), wb=op.workspace(True))
        s.update({n: op.out() for n in ("Y", "Z", "dz")}, dX=torch.empty_like(op.X), dW=[torch.empty_like(w) for w in op.w], db=torch.empty_like(s["bias"]))
        state.append(s)

    def step(op, s):
        osdp.osdp_split_linear_fwd_epilogue(op.X, op.w, s["Y"], op.k, s["ws"], plan=op.plan, stream_compute=s["stream"],
                                            epilogue=osdp.Epilogue(bias=s["bias"], activation=ACTS["gelu"], residual=s["residual"], z=s["Z"]))
        osdp.osdp_split_linear_bwd_epilogue(op.X, s["dY"], op.w, s["dX"], s["dW"], op.k, s["wb"], plan=op.plan, stream_compute=s["stream"],
                                            epilogue=osdp.EpilogueGrad(activation=ACTS["gelu"], z=s["Z"], dz=s["dz"], dbias=s["db"]))

    def outputs(s):
        return [t.clone() for t in (s["Y"], s["Z"], s["dz"], s["dX"], s["db"], *s["dW"])]

    torch.cuda.synchronize()
    want = []
    for op, s in zip(ops, state):
        step(op, s)
        torch.cuda.synchronize()
        want.append(outputs(s))
    wrong = []

    def work(i):
        try:
            for _ in range(50):
                step(ops[i], state[i])
        except Exception as e:  # noqa: BLE001 (whatever it is, the test's own thread says it)
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
    for s, w in zip(state, want):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outputs(s), w))


class OnlyPython:
    """In the place of the binding's way through C: nothing is answered there."""
    linear = qk = staticmethod(lambda *a: None)


@pytest.mark.parametrize("T,ld", [(1, 0), (40, 0), (40, 24), (300, 8)])
@pytest.mark.parametrize("parts", [(), ("bias", "residual", "z"), ("bias",), ("z",)])
def test_both_ways_into_the_library_hand_over_the_same(monkeypatch, T, ld, parts):
    """Tensors are looked at in C, or in Python where that gives no answer: the same bits, for rows of any length and parts left out."""
    I, O, N, k = 264, 520, 3, 1
    op, given = Op(T, I, O, N, k), []
    wide = lambda cols, seed: rand(T, cols + ld, seed=seed)[:, :cols]  # noqa: E731
    op.X, residual, dY = wide(I, 1), wide(O, 2), wide(O, 3)
    for way in ("C", "Python"):
        if way == "Python":
            monkeypatch.setattr(osdp.binding, "_calls", OnlyPython)
        bias = rand(O, seed=4, dtype=torch.float32) if "bias" in parts else None
        act = ACTS["gelu"] if "z" in parts else ACTS["none"]
        Y, Z, dz = (torch.full((T, O + ld), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :O] for _ in range(3))
        op.fwd(Y, bias=bias, activation=act, residual=residual if "residual" in parts else None, z=Z if "z" in parts else None)
        db = None if bias is None else torch.full_like(bias, float("nan"))
        dX, dW = op.bwd(dY, activation=act, z=Z if "z" in parts else None, dz=dz if "z" in parts else None, dbias=db)
        given.append([t.clone() for t in (Y, Z, dz, dX, dW)] + ([] if db is None else [db]))
    assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(*given))
