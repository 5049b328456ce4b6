"""The operator in 8-bit integers against plain arithmetic.

The whole numbers and their sums are exact, and the two scalings and the rounding of the result are the same three fp32
roundings on either side, so everything is compared bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2209_13258_amd as osdp
import workloads as wl

pytestmark = pytest.mark.gpu


def widen(bits):
    return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32)


def to_8_bits(x, axis):
    """(whole numbers, fp32 scale) along an axis, from the definition, in 64 bits."""
    a = np.abs(x.astype(np.float64)).max(axis=axis, keepdims=True)
    fine = np.isfinite(a)
    at = np.where(fine & (a > 0), a, 1.0)
    with np.errstate(invalid="ignore"):
        t = np.floor(np.abs(x.astype(np.float64)) * 127 / at + 0.5)
        q = np.where(fine & (a > 0), np.sign(x) * t, 0.0)
    scale = np.where(fine, a.astype(np.float32) / np.float32(127), np.float32(np.nan)).astype(np.float32)
    return np.nan_to_num(q).astype(np.int64), scale.reshape(-1)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def cut(flat, N, dtype, fill):
    L = -(-flat.size // N)
    out = torch.full((N * L,), fill, dtype=dtype)
    out[:flat.size] = torch.from_numpy(flat)
    return [out[s * L:(s + 1) * L].clone().cuda() for s in range(N)]


def expected(x, q, scale):
    """Y as fp32 values that bf16 holds: the sums exactly, then as the kernels round."""
    xq, xs = to_8_bits(x, 1)
    sums = (xq.astype(np.float64) @ q.T.astype(np.float64)).astype(np.int64)  # (below 2^53: exact)
    with np.errstate(invalid="ignore", over="ignore"):
        y = sums.astype(np.float32) * xs[:, None] * scale[None, :]
    return torch.from_numpy(y).to(torch.bfloat16).float().numpy()


class Weight:
    def __init__(self, I, O, N, seed=0):
        g = np.random.default_rng([seed, I, O, N])
        self.I, self.O, self.N = I, O, N
        self.q = np.clip(np.rint(g.standard_normal((O, I)) * 40), -127, 127).astype(np.int8)
        self.scale = (np.exp(g.standard_normal(O)) * 1e-3).astype(np.float32)
        self.shards = cut(self.q.reshape(-1), N, torch.int8, 99)
        self.dev_scale = torch.from_numpy(self.scale).cuda()


def tokens(T, I, seed=0):
    x = np.random.default_rng([seed, T, I]).standard_normal((T, I)).astype(np.float32)
    x *= np.exp(np.random.default_rng([seed, T]).standard_normal((T, 1))).astype(np.float32)
    return bf16(x).float().numpy()


def forward(w, x, k=1, pad_x=0, pad_y=0, stream=None, out=None):
    T = x.shape[0]
    X = torch.full((T, w.I + pad_x), float("nan"), dtype=torch.bfloat16, device="cuda")
    X[:, :w.I] = bf16(x).cuda()
    Y = torch.full((T + 1, w.O + pad_y), 3.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    need, _ = osdp.osdp_split_linear_i8_workspace_bytes(T, w.I, w.O, w.N, k)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    osdp.osdp_split_linear_i8_fwd(X[:, :w.I], w.shards, w.dev_scale, Y[:T, :w.O], k, ws[:need], stream=stream)
    torch.cuda.synchronize()
    y = Y.float().cpu().numpy()
    assert (y[T:] == 3.0).all() and (y[:, w.O:] == 3.0).all(), "rows behind the last token or columns behind the last channel were written"
    assert (ws[need:] == 255).all(), "written behind the workspace"
    return y[:T, :w.O]


def same(got, want):
    assert got.shape == want.shape
    bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{int(bad.sum())} of {bad.size} differ, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


TOKENS = [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 127, 128, 129, 160, 200, 255, 256, 257, 300, 500, 513]


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("I,O,N", [(256, 1024, 2), (1040, 520, 4), (4096, 264, 1)])
def test_product_over_token_counts(T, I, O, N):
    print("int8 product", T, I, O, N, flush=True)
    w, x = Weight(I, O, N), tokens(T, I)
    same(forward(w, x), expected(x, w.q, w.scale))


@pytest.mark.parametrize("T", [1, 9, 40, 70, 140, 300])
@pytest.mark.parametrize("I,O,N,k", [(16, 8, 1, 1), (16, 1024, 64, 2), (48, 24, 4, 3), (112, 40, 5, 5), (128, 136, 1, 0), (144, 80, 16, 2),
                                     (2064, 264, 3, 3), (8208, 48, 9, 1), (32, 2056, 16, 1), (336, 1000, 3, 5), (16384, 72, 8, 1),
                                     (4096, 24, 64, 1), (640, 2600, 8, 1), (512, 264, 8, 1), (272, 3000, 24, 1)])
def test_product_over_weight_shapes_and_cuts(T, I, O, N, k):
    """Row blocks of channels, flat cuts inside a channel's row, shards shorter than a row, narrow and long ones."""
    print("int8 product", T, I, O, N, k, flush=True)
    w, x = Weight(I, O, N), tokens(T, I)
    same(forward(w, x, k), expected(x, w.q, w.scale))


@pytest.mark.parametrize("T", [16, 17, 32, 33, 47, 48, 49, 63, 64])
@pytest.mark.parametrize("I,O,N", [(336, 1000, 21), (4096, 520, 16), (2048, 40, 64)])
def test_rows_that_run_over_the_ends_of_shards(T, I, O, N):
    print("int8 product", T, I, O, N, flush=True)
    w, x = Weight(I, O, N), tokens(T, I)
    same(forward(w, x, pad_y=8), expected(x, w.q, w.scale))


@pytest.mark.parametrize("T,I,O,N", [(1, 4096, 2056, 1), (1, 12288, 1024, 8), (2, 8192, 4104, 8), (9, 4096, 1032, 16), (40, 4096, 520, 16), (33, 4096, 8192, 8),
                                     (64, 8192, 2048, 2), (100, 8192, 3000, 8), (128, 16384, 1024, 4), (129, 4096, 2048, 8), (250, 16384, 2048, 4),
                                     (5, 131072, 72, 1), (60, 20480, 1000, 5)])
def test_rows_a_multiple_of_4_kb_apart(T, I, O, N):
    """Workgroups that begin at different places of the reduction, with and without parts."""
    print("int8 product", T, I, O, N, flush=True)
    w, x = Weight(I, O, N), tokens(T, I)
    same(forward(w, x), expected(x, w.q, w.scale))


# one that each of the kernels is chosen for, with the parts that its tiles' reductions are cut into
CHOICES = [((5, 512, 512, 8), "i8_fused_kernel", 1), ((512, 512, 512, 8), "i8_fused_kernel", 1), ((30, 2048, 1024, 8), "i8_few_kernel", 1), ((300, 1152, 2048, 8), "i8_w4_kernelILi2ELi2ELi4", 1),
           ((161, 14448, 960, 8), "i8_w4_kernelILi2ELi2ELi4", 4), ((1000, 4096, 4096, 4), "i8_w4_kernelILi4ELi4ELi4", 1),
           ((300, 16384, 2048, 4), "i8_w4_kernelILi4ELi4ELi4", 4), ((500, 2560, 10240, 8), "i8_w4_kernelILi4ELi4ELi2", 1),
           ((1500, 1024, 16424, 8), "i8_w4_kernelILi8ELi8ELi2", 1)]


@pytest.mark.parametrize("sizes,kernel,parts", CHOICES)
def test_every_kernel_gives_the_same_whole_numbers(sizes, kernel, parts):
    import gpu_harness as H
    T, I, O, N = sizes
    print("int8 product", *sizes, kernel, flush=True)
    w, x = Weight(I, O, N), tokens(T, I)
    want = expected(x, w.q, w.scale)
    same(forward(w, x), want)
    X, Y = bf16(x).cuda(), torch.zeros(T, O, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, 1)[0], dtype=torch.uint8, device="cuda")
    ran = H.kernels(lambda s: osdp.osdp_split_linear_i8_fwd(X, w.shards, w.dev_scale, Y, 1, ws, stream=s))
    assert len(ran) == (1 if kernel == "i8_fused_kernel" else 2) and kernel in ran[-1][0], ran
    if parts > 1:  # more workgroups than tiles, and the same numbers every time, whichever part arrives last
        side = 64 if "ILi2ELi2" in ran[-1][0] else 128
        assert ran[-1][1] >= 2 * -(-T // side) * N * -(-(O // N) // side)
        for _ in range(20):
            Y.zero_()
            osdp.osdp_split_linear_i8_fwd(X, w.shards, w.dev_scale, Y, 1, ws)
            torch.cuda.synchronize()
            same(Y.float().cpu().numpy(), want)


@pytest.mark.parametrize("T,I,O,N", [(1, 32768, 1024, 8), (33, 131072, 128, 2), (1030, 1024, 2048, 8), (700, 8192, 776, 1), (2100, 384, 3080, 8),
                                     (4096, 256, 5000, 5), (4096, 256, 5000, 16), (4000, 1024, 1000, 8), (3000, 512, 2560, 8)])
def test_larger_products(T, I, O, N):
    print("int8 product", T, I, O, N, flush=True)
    w, x = Weight(I, O, N), tokens(T, I)
    same(forward(w, x), expected(x, w.q, w.scale))


@pytest.mark.parametrize("T", [1, 5, 33, 130, 400])
def test_strides(T):  # (in place, and from T = 400 on gathered)
    w, x = Weight(528, 392, 11), tokens(T, 528)
    want = expected(x, w.q, w.scale)
    for pad_x, pad_y in ((8, 0), (0, 8), (1000, 24)):
        same(forward(w, x, pad_x=pad_x, pad_y=pad_y), want)


@pytest.mark.parametrize("T", [1, 4, 20, 70, 150, 300, 3000])
def test_slices_and_shards_do_not_change_a_bit(T):
    I, O = 336, 1000
    x = tokens(T, I)
    base = Weight(I, O, 1)
    want = forward(base, x)
    same(want, expected(x, base.q, base.scale))
    for N, k in ((8, 1), (3, 1), (3, 5), (7, 25), (21, 125), (40, 5)):
        w = Weight(I, O, N)
        w.q, w.scale, w.dev_scale = base.q, base.scale, base.dev_scale
        w.shards = cut(base.q.reshape(-1), N, torch.int8, 99)
        same(forward(w, x, k), want)


@pytest.mark.parametrize("T", [7, 70, 200])
def test_tokens_that_are_zeros_or_hold_no_numbers(T):
    w, x = Weight(272, 264, 2), tokens(T, 272)
    x[0] = 0
    x[1, 5] = np.inf
    x[2, 271] = np.nan
    x[3, 0] = -np.inf
    x[4] = 0
    x[4, 100] = 2.0 ** -133                    # the smallest bf16
    x[5] = bf16(x[5] * 2.0 ** -125).float().numpy()  # below fp32's normal range, mostly
    x[6] = np.where(np.arange(272) % 2, 3.3895313892515355e38, -1.0)
    got = forward(w, x)
    same(got, expected(x, w.q, w.scale))
    assert (got[0] == 0).all() and np.isnan(got[1:4]).all() and np.isfinite(got[4:6]).all()


def _few_columns(X, shards, scale, O, rows, cols):
    """Y at some rows and columns, from the definition, in 64 bits on the GPU."""
    I = X.shape[1]
    x = X[rows].float().cpu().numpy()
    L = shards[0].numel()
    q = np.stack([np.concatenate([shards[s][a:b].cpu().numpy() for s, a, b in _pieces(c * I, I, L)]) for c in cols])
    return expected(x, q, scale[cols].cpu().numpy())


def _pieces(start, length, L):
    """(shard, from, to) of the pieces that a run of a flat matrix lies in."""
    out = []
    while length > 0:
        s, a = divmod(start, L)
        b = min(L, a + length)
        out.append((s, a, b))
        start, length = start + b - a, length - (b - a)
    return out


@pytest.mark.parametrize("T,I,O,N", [(2, 131072, 40000, 5), (70, 131072, 40000, 5), (300, 131072, 33000, 16)])
def test_weights_of_more_than_32_bits(T, I, O, N):
    """5 GB of weights: whole channels in five shards of more than 2^29 bytes, and cut within channels in sixteen."""
    print("int8 product", T, I, O, N, flush=True)
    L = -(-I * O // N)
    gen = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randint(-127, 128, (1000003,), dtype=torch.int8, device="cuda", generator=gen)
    shards = [base.roll(s).repeat(-(-L // 1000003))[:L].contiguous() for s in range(N)]
    scale = torch.rand(O, device="cuda", generator=gen) * 1e-3
    X = torch.randn(T, I, device="cuda", generator=gen).to(torch.bfloat16)
    Y = torch.zeros(T, O, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, 1)[0], dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_fwd(X, shards, scale, Y, 1, ws)
    torch.cuda.synchronize()
    rows = [0, T // 2, T - 1]
    cols = [0, 1, O // 3, (1 << 31) // I - 1, (1 << 31) // I, (1 << 32) // I - 1, (1 << 32) // I, O - 1]
    same(Y[rows][:, cols].float().cpu().numpy(), _few_columns(X, shards, scale, O, rows, cols))


@pytest.mark.parametrize("T,I,O,N", [(1, 16, (1 << 27) + 64, 1), (5, 16, (1 << 27) + 64, 8), (3, 48, (1 << 27) + 8, 3), (2, 16, (1 << 31) - 512, 1)])
def test_most_channels(T, I, O, N):
    """More channels than a launch of the kernels for few tokens has threads for."""
    print("int8 product", T, I, O, N, flush=True)
    L = -(-I * O // N)
    gen = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randint(-127, 128, (1000003,), dtype=torch.int8, device="cuda", generator=gen)
    shards = [base.roll(s).repeat(-(-L // 1000003))[:L].contiguous() for s in range(N)]
    scale = (torch.rand(1000, device="cuda", generator=gen) * 1e-3).repeat(-(-O // 1000))[:O].contiguous()
    X = torch.randn(T, I, device="cuda", generator=gen).to(torch.bfloat16)
    Y = torch.zeros(T, O, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, 1)[0], dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_fwd(X, shards, scale, Y, 1, ws)
    torch.cuda.synchronize()
    rows = sorted({0, T - 1})
    cols = [0, 1, 255, 256, O // N - 1, O // N % O, O // N % O + 1, O // 3, (1 << 27) - 17, (1 << 27) - 1, 1 << 27, O - 9, O - 1]
    assert all(0 <= c < O for c in cols)
    same(Y[rows][:, cols].float().cpu().numpy(), _few_columns(X, shards, scale, O, rows, cols))


def test_tokens_of_more_than_32_bits():
    """4.9 GB of rounded tokens, 9.8 GB in bf16."""
    T, I, O, N = 300000, 16384, 16, 1
    print("int8 product", T, I, O, N, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = Weight(I, O, N)
    X = torch.randn(1000, I, device="cuda", generator=gen).to(torch.bfloat16).repeat(300, 1)
    Y = torch.zeros(T, O, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, 1)[0], dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_fwd(X, w.shards, w.dev_scale, Y, 1, ws)
    torch.cuda.synchronize()
    want = expected(X[:1000].float().cpu().numpy(), w.q, w.scale)
    for a in range(0, T, 1000):
        assert torch.equal(Y[a:a + 1000], Y[:1000]), a
    same(Y[:1000].float().cpu().numpy(), want)


def test_weight_of_more_than_32_bits_to_8():
    I, O, N = 131072, 40000, 5
    print("int8 quantize", I, O, N, flush=True)
    L = I * O // N
    gen = torch.Generator(device="cuda").manual_seed(3)
    base = (torch.randn(1000003, device="cuda", generator=gen) * 0.02).to(torch.bfloat16)
    W = [base.roll(s).repeat(-(-L // 1000003))[:L].contiguous() for s in range(N)]
    q = [torch.zeros(L, dtype=torch.int8, device="cuda") for _ in range(N)]
    scale = torch.zeros(O, device="cuda")
    ws = torch.empty(osdp.osdp_split_linear_i8_quantize_workspace_bytes(I, O, N), dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_quantize(I, O, W, q, scale, ws)
    torch.cuda.synchronize()
    full = torch.cat(W).view(I, O)
    for c in (0, 1, 16383, 16384, 32767, 32768, O - 1):
        want, want_scale = to_8_bits(full[:, c:c + 1].float().cpu().numpy(), 0)
        s, off = c * I // L, c * I % L
        assert np.array_equal(q[s][off:off + I].cpu().numpy(), want[:, 0]) and scale[c].item() == want_scale[0], c


def test_extreme_sums_stay_exact():
    """Every number at its largest: 131072 * 127 * 127 = 2113929216 is below 2^31."""
    I, O = 131072, 32
    w = Weight(I, O, 1)
    w.q = np.full((O, I), 127, np.int8)
    w.q[1::2] = -127
    w.scale = np.full(O, 1.0, np.float32)
    w.dev_scale, w.shards = torch.from_numpy(w.scale).cuda(), cut(w.q.reshape(-1), 1, torch.int8, 0)
    for T in (1, 20, 70, 130):
        x = np.full((T, I), 127.0, np.float32)
        got = forward(w, x)
        same(got, expected(x, w.q, w.scale))
        assert got[0, 0] == 2113929216 // 2 ** 24 * 2 ** 24


def test_halves_go_away_from_zero():
    """Quotients of all significands by every sixteenth largest one, at eight powers of two: none may be taken for the other side of a half."""
    a = np.arange(128, 256)
    for b in range(128, 256):
        x = np.zeros((8, 144), np.float32)
        for j in range(8):
            x[j, :128] = a * 2.0 ** -j
            x[j, 128] = b * 2.0 if j == 0 else b * 1.0
            x[j, 129:] = -x[j, :15]
        x[0] = np.where(np.abs(x[0]) > b * 2.0, 0, x[0])
        x[1:] = np.where(np.abs(x[1:]) > b, 0, x[1:])
        if b % 16:
            continue
        I = 144
        w = Weight(I, I, 1)
        w.q = (np.eye(I) * 127).astype(np.int8)     # Y = xq * 127 * scales: the rounded numbers themselves
        w.scale = np.full(I, 1.0 / 127, np.float32)
        w.dev_scale, w.shards = torch.from_numpy(w.scale).cuda(), cut(w.q.reshape(-1), 1, torch.int8, 0)
        same(forward(w, x), expected(x, w.q, w.scale))


def quantize(W, I, O, N):
    shards = cut(W.view(torch.int16).numpy().reshape(-1), N, torch.int16, 0x7FC0)
    shards = [s.view(torch.bfloat16) for s in shards]
    L = -(-I * O // N)
    q = [torch.full((L,), 99, dtype=torch.int8, device="cuda") for _ in range(N)]
    scale = torch.full((O + 4,), 7.0, device="cuda")
    ws = torch.full((osdp.osdp_split_linear_i8_quantize_workspace_bytes(I, O, N) + 256,), 255, dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_quantize(I, O, shards, q, scale[:O], ws[:-256])
    torch.cuda.synchronize()
    flat = torch.cat(q).cpu().numpy()
    assert (flat[I * O:] == 99).all() and (scale[O:] == 7.0).all() and (ws[-256:] == 255).all()
    return flat[:I * O].reshape(O, I), scale[:O].cpu().numpy(), q, scale[:O]


@pytest.mark.parametrize("I,O,N", [(16, 8, 1), (16, 16, 16), (32, 24, 3), (64, 40, 8), (128, 128, 2), (144, 136, 4), (256, 1024, 2), (272, 264, 11),
                                   (1040, 520, 5), (2560, 1280, 8), (4096, 8, 64), (16, 4096, 64), (336, 1000, 3), (131072, 16, 8), (1024, 4096, 8), (1008, 1032, 7),
                                   (1040, 72, 2), (2048, 136, 4), (16, 8, 8), (512, 8, 64), (20016, 536, 3)])
def test_weight_to_8_bits(I, O, N):
    print("int8 quantize", I, O, N, flush=True)
    g = np.random.default_rng([I, O])
    W = bf16(g.standard_normal((I, O)) * 0.02 * np.exp(g.standard_normal(O)))
    W[:, 0] = 0
    W[I // 2, 1] = float("inf")
    W[I - 1, 2] = float("nan")
    W[:, 3] = bf16(W[:, 3].float().numpy() * 2.0 ** -124)
    W[0, 4] = W[:, 4].float().abs().max() * 2    # half of it is a half
    W[1, 4] = W[0, 4] / 2
    W[2, 4] = -W[0, 4] / 2
    got, scale, _, _ = quantize(W, I, O, N)
    want, want_scale = to_8_bits(W.float().numpy(), 0)
    assert np.array_equal(got, want.T)
    assert np.array_equal(scale, want_scale, equal_nan=True)
    assert got[4, 1] == 64 and got[4, 2] == -64 and np.isnan(scale[1]) and np.isnan(scale[2]) and scale[0] == 0


def test_shards_are_looked_at_before_their_addresses_are_taken():
    """Tensors as a program may have them: views, parameters, several dimensions; and those that do not do."""
    look = osdp.binding._checked_pointers
    z = lambda *n, d=torch.int8: torch.zeros(*n, dtype=d, device="cuda")  # noqa: E731
    flat, weight = z(4096), torch.nn.Parameter(z(64, 8, d=torch.bfloat16))
    good = [z(1024), flat[7:1031], flat.view(4, 1024)[1], flat.view(torch.uint8)[:1024], z(8, 1, 128), z(1, 1024).t()]
    bits8, bf16 = bytes((0, 8, 1, 8)), bytes((4, 16))
    out = look(good, 1024, bits8, 0)
    assert np.frombuffer(out, np.uint64).tolist() == [t.data_ptr() for t in good]
    assert np.frombuffer(look([weight, weight.detach()], 1024, bf16, 0), np.uint64).tolist() == [weight.data_ptr()] * 2
    for bad in (z(1023), flat[::2], flat.view(64, 64).t(), z(1).expand(1024), z(1024, d=torch.bfloat16), z(1024, d=torch.int16), z(1024).cpu(),
                z(1024, d=torch.bool)):
        for place in range(2):
            ts = [z(1024), z(1024)]
            ts[place] = bad
            assert look(ts, 1024, bits8, 0) is None
            w = [z(1024, d=torch.bfloat16) for _ in range(2)]
            with pytest.raises(osdp.OsdpError, match=r"q_shards\[%d\]" % place):
                osdp.osdp_split_linear_i8_quantize(64, 32, w, ts, z(32, d=torch.float32), z(1 << 16, d=torch.uint8))
    for bad in (z(1024, d=torch.float32), z(1024, d=torch.float16), z(511, d=torch.bfloat16)):
        with pytest.raises(osdp.OsdpError, match="w_shards"):
            osdp.osdp_split_linear_i8_quantize(64, 32, [z(1024, d=torch.bfloat16), bad], [z(1024), z(1024)], z(32, d=torch.float32), z(1 << 16, d=torch.uint8))
    assert look([z(1024)], 1024, bits8, 1) is None


def test_graph_of_two_products_sharing_a_workspace():
    """Captured one after another on one stream, replayed with other inputs and the program's own work between."""
    a, b = Weight(512, 768, 8), Weight(768, 520, 5)
    for T in (3, 90):
        need = max(osdp.osdp_split_linear_i8_workspace_bytes(T, w.I, w.O, w.N, 1)[0] for w in (a, b))
        ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        X = torch.zeros(T, 512, dtype=torch.bfloat16, device="cuda")
        H = torch.zeros(T, 768, dtype=torch.bfloat16, device="cuda")
        Y = torch.zeros(T, 520, dtype=torch.bfloat16, device="cuda")
        stream = torch.cuda.Stream()

        def both():
            osdp.osdp_split_linear_i8_fwd(X, a.shards, a.dev_scale, H, 1, ws, stream=stream)
            osdp.osdp_split_linear_i8_fwd(H, b.shards, b.dev_scale, Y, 1, ws, stream=stream)
        torch.cuda.synchronize()
        both()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            both()
        for k in range(4):
            x = tokens(T, 512, seed=k)
            X.copy_(bf16(x))
            ws.fill_(255)
            Y.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            h = expected(x, a.q, a.scale)
            same(H.float().cpu().numpy(), h)
            same(Y.float().cpu().numpy(), expected(h, b.q, b.scale))


def test_two_streams_with_their_own_workspaces():
    w = Weight(1024, 2048, 8)
    xs = [tokens(T, 1024, seed=T) for T in (64, 200)]
    X = [bf16(x).cuda() for x in xs]
    Y = [torch.zeros(x.shape[0], 2048, dtype=torch.bfloat16, device="cuda") for x in xs]
    ws = [torch.zeros(osdp.osdp_split_linear_i8_workspace_bytes(x.shape[0], 1024, 2048, 8, 1)[0], dtype=torch.uint8, device="cuda") for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            osdp.osdp_split_linear_i8_fwd(X[i], w.shards, w.dev_scale, Y[i], 1, ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for x, y in zip(xs, Y):
        same(y.float().cpu().numpy(), expected(x, w.q, w.scale))


def test_a_training_step_and_its_answer_in_8_bits():
    """The operators as they are used: forward and backward of the split operator, the norm of the gradients, the step on
    the shards, the 8-bit weight from them, and its product."""
    T, I, O, N, k = 200, 256, 1024, 2, 4
    d = wl.small_case(5, T, I, O, N, w_std=0.02)
    import gpu_harness as H
    op = H.Operator(d["X"], d["dY"], d["W_shards"], O)
    masters = [s.float() for s in op.W]
    m, v = ([torch.zeros(op.L, dtype=torch.uint8, device="cuda") for _ in range(N)] for _ in range(2))
    exps = [torch.zeros(2 * -(-op.L // 128), dtype=torch.uint8, device="cuda") for _ in range(N)]
    table = osdp.AdamWTable(params=op.W, grads=op.dW, masters=masters, m=m, v=v, exps=exps, weight_decay=0.1)
    sumsq = torch.zeros(1, dtype=torch.float64, device="cuda")
    ws = torch.zeros(max(256, osdp.osdp_adamw_grad_sumsq_workspace_bytes(table)), dtype=torch.uint8, device="cuda")
    start = [w.clone() for w in masters]
    op.fwd(k)
    op.bwd(k)
    osdp.osdp_adamw_grad_sumsq(table, sumsq, ws)
    osdp.osdp_adamw_step(table, lr=1e-3, step=1, grad_sumsq=sumsq, max_norm=1.0, seed=1)
    torch.cuda.synchronize()
    dW = H.widen(d["X"]).T @ H.widen(d["dY"])
    assert abs(float(sumsq.sqrt()) / np.linalg.norm(dW) - 1) < 2.0 ** -8  # (the gradients are rounded to bf16)
    moved = torch.cat(masters) - torch.cat(start) * (1 - 1e-3 * 0.1)
    # the first step of Adam is lr in the direction against the gradient, where eps is nothing beside it
    sure = torch.cat([g.float().abs() for g in op.dW]) > 1e-2
    clip = 1.0 / float(sumsq.sqrt())
    big = sure & (torch.cat([g.float().abs() for g in op.dW]) * clip > 1e-5)
    assert ((moved / -1e-3 - torch.cat([g.float().sign() for g in op.dW]))[big].abs() < 2e-3).all()
    W = torch.cat(op.W)[:I * O].view(I, O).cpu()
    q = [torch.zeros(op.L, dtype=torch.int8, device="cuda") for _ in range(N)]
    scale = torch.zeros(O, device="cuda")
    qws = torch.zeros(osdp.osdp_split_linear_i8_quantize_workspace_bytes(I, O, N), dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_quantize(I, O, op.W, q, scale, qws)
    Y = torch.zeros(T, O, dtype=torch.bfloat16, device="cuda")
    lws = torch.zeros(osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, k)[0], dtype=torch.uint8, device="cuda")
    osdp.osdp_split_linear_i8_fwd(op.X, q, scale, Y, k, lws)
    torch.cuda.synchronize()
    want_q, want_scale = to_8_bits(W.float().numpy(), 0)
    same(Y.float().cpu().numpy(), expected(widen(d["X"]), want_q.T, want_scale))
    # against the product without 8 bits: two roundings of half a step each, of 127 to the largest magnitude
    exact = widen(d["X"]).astype(np.float64) @ W.double().numpy()
    ax, aw = np.abs(widen(d["X"])).max(1)[:, None].astype(np.float64), W.double().abs().numpy().max(0)[None, :]
    bound = (ax / 254) * np.abs(W.double().numpy()).sum(0)[None, :] + (aw / 254) * np.abs(widen(d["X"]).astype(np.float64)).sum(1)[:, None] + I * ax * aw / 254 ** 2
    y = Y.double().cpu().numpy()
    assert (np.abs(y - exact) <= bound + 2.0 ** -8 * np.abs(exact) + 2.0 ** -8 * bound).all()
