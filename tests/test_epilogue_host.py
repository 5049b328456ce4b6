"""Bias, activation and residual around the operator, and norms and rotation of queries and keys: formulas, sizes and refusals,
which need no GPU."""
import ctypes
import math
import random

import pytest
import torch

import epilogue_reference as R
import paper_2209_13258_amd as osdp
from paper_2209_13258_amd import binding as B

P = 1 << 24  # an aligned address that nothing here follows; matrices lie P apart
INVALID, UNSUPPORTED, WORKSPACE = B.OSDP_ERR_INVALID_ARG, B.OSDP_ERR_UNSUPPORTED, B.OSDP_ERR_WORKSPACE
T, I, O = 16, 64, 128


# ---- the references that the kernels are tested against -----------------------------------------------------------
@pytest.mark.parametrize("name", R.NAMES)
def test_slopes_are_the_differences_of_the_activations(name):
    z = torch.linspace(-9, 9, 3601, dtype=torch.float64)
    z = z[(z.abs() > 1e-3)]  # (relu has no slope at 0)
    h = 1e-5
    d = (R.act(name, z + h) - R.act(name, z - h)) / (2 * h)
    # central differences: h^2 / 6 of the third derivative (below 3 for all of them), and 2^-53 of values up to 9 over h
    assert (d - R.slope(name, z)).abs().max() < h * h * 3 + 9 * 2.0 ** -52 / h
    assert torch.allclose(R.act(name, z), {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
                                           "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh"),
                                           "silu": torch.nn.functional.silu}[name](z), rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_the_pass_back_is_the_gradient_of_the_pass_forward(norm, interleaved):
    g = torch.Generator().manual_seed(5)
    x, dy = (torch.randn(3, 2, 24, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(24, generator=g, dtype=torch.float64) if norm else None
    freqs, pos = torch.rand(8, generator=g, dtype=torch.float64), torch.tensor([0, 5, 100000])
    x.requires_grad_()
    if norm:
        w.requires_grad_()
    y = R.qk(x, pos, freqs, w, 1e-6, norm, interleaved)
    grads = torch.autograd.grad((y * dy).sum(), [x, w] if norm else [x])
    dx, dw = R.qk_back(x.detach(), dy, pos, freqs, None if w is None else w.detach(), 1e-6, norm, interleaved)
    assert torch.allclose(grads[0], dx, rtol=1e-10, atol=1e-12)
    assert not norm or torch.allclose(grads[1], dw, rtol=1e-10, atol=1e-12)
    # and of its differences along a direction
    u, h = torch.randn(x.shape, generator=g, dtype=torch.float64), 1e-6
    f = [(R.qk(x.detach() + s * h * u, pos, freqs, w, 1e-6, norm, interleaved) * dy).sum().item() for s in (1, -1)]
    assert abs((f[0] - f[1]) / (2 * h) - (dx * u).sum().item()) < 1e-6


# ---- the operator with an epilogue --------------------------------------------------------------------------------
def shards(n, at=8 * P):
    return (ctypes.c_void_p * n)(*[at + i * P for i in range(n)])


def forward(shape=(T, I, O, 2, 1), x=P, ldx=I, y=2 * P, ldy=O, ws=4 * P, ws_bytes=1 << 40, epilogue=True, **more):
    e = B.osdp_epilogue(3 * P, 5 * P, O, 6 * P, O, B.OSDP_ACT_GELU, B.OSDP_BF16)
    for k, v in more.items():
        setattr(e, k, v)
    return osdp.lib.osdp_split_linear_fwd_epilogue(ctypes.byref(B.osdp_shape(*shape)), None, 0, ctypes.byref(e) if epilogue else None,
                                                   x, ldx, shards(shape[3]), None, 0, y, ldy, ws, ws_bytes, None, None)


def backward(shape=(T, I, O, 2, 1), x=P, dy=2 * P, lddy=O, dx=3 * P, ws=4 * P, ws_bytes=1 << 40, epilogue=True, **more):
    e = B.osdp_epilogue_grad(5 * P, O, 6 * P, O, 7 * P, B.OSDP_ACT_GELU, B.OSDP_BF16)
    for k, v in more.items():
        setattr(e, k, v)
    return osdp.lib.osdp_split_linear_bwd_epilogue(ctypes.byref(B.osdp_shape(*shape)), None, 0, ctypes.byref(e) if epilogue else None,
                                                   x, I, dy, lddy, shards(shape[3]), None, 0, dx, I, shards(shape[3], 32 * P), None, ws,
                                                   ws_bytes, None, None)


def passes_the_checks(status):
    """Whether a call got as far as asking for the device, which is not there (or, where there is one, was not made)."""
    return status not in (INVALID, UNSUPPORTED, WORKSPACE) or b"device" in osdp.lib.osdp_last_error()


@pytest.fixture
def no_gpu():
    if torch.cuda.is_available():
        pytest.skip("calls with made-up addresses would run")


@pytest.mark.parametrize("more,status", [
    (dict(epilogue=False), INVALID), (dict(activation=-1), INVALID), (dict(activation=5), INVALID), (dict(bias_type=2), INVALID),
    (dict(bias=3 * P + 8), UNSUPPORTED), (dict(residual=5 * P + 8), UNSUPPORTED), (dict(z=6 * P + 2), UNSUPPORTED),
    (dict(ld_residual=O - 8), INVALID), (dict(ldz=O - 8), INVALID), (dict(ldz=O + 4), UNSUPPORTED), (dict(ld_residual=O + 4), UNSUPPORTED),
    (dict(z=2 * P), INVALID), (dict(z=2 * P + 16), INVALID), (dict(residual=2 * P + 16), INVALID), (dict(residual=2 * P, ld_residual=2 * O), INVALID),
    (dict(z=5 * P), INVALID), (dict(z=P), INVALID), (dict(y=P), INVALID), (dict(bias=2 * P), INVALID), (dict(bias=6 * P + 32), INVALID),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(ldx=I - 8), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=0), WORKSPACE),
    (dict(shape=(T, I, O, 0, 1)), INVALID), (dict(shape=(-1, I, O, 1, 1)), INVALID), (dict(shape=(T, I, O + 4, 1, 1)), INVALID),
    (dict(shape=(T, 60, O, 1, 1)), UNSUPPORTED)])
def test_forward_refuses(more, status):
    assert forward(**more) == status
    assert osdp.lib.osdp_last_error()


@pytest.mark.parametrize("more", [
    dict(), dict(residual=2 * P), dict(bias=None, residual=None, z=None, activation=0), dict(shape=(0, I, O, 2, 1), x=None, y=None),
    dict(y=2 * P, ldy=3 * O, residual=2 * P + 2 * O, ld_residual=3 * O, z=2 * P + 4 * O, ldz=3 * O), dict(bias_type=B.OSDP_F32)])
def test_forward_takes(no_gpu, more):
    """A residual that is Y, parts of one wide matrix side by side, no tokens."""
    assert passes_the_checks(forward(**more))


@pytest.mark.parametrize("more,status", [
    (dict(epilogue=False), INVALID), (dict(activation=9), INVALID), (dict(bias_type=-1), INVALID), (dict(dbias=7 * P + 4), UNSUPPORTED),
    (dict(z=None), INVALID), (dict(dz=None), INVALID), (dict(activation=0), INVALID), (dict(ldz=O - 8), INVALID), (dict(lddz=O + 2), UNSUPPORTED),
    (dict(dz=2 * P, lddz=2 * O), INVALID), (dict(dz=2 * P + 16), INVALID), (dict(dz=5 * P + 16), INVALID), (dict(dz=P), INVALID),
    (dict(dbias=2 * P), INVALID), (dict(dbias=3 * P), INVALID), (dict(dbias=6 * P + 64), INVALID), (dict(dbias=P), INVALID),
    (dict(dy=None), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=0), WORKSPACE)])
def test_backward_refuses(more, status):
    assert backward(**more) == status
    assert osdp.lib.osdp_last_error()


@pytest.mark.parametrize("more", [dict(), dict(dz=2 * P), dict(dz=5 * P), dict(activation=0, z=None, dz=None), dict(dbias=None),
                                  dict(shape=(0, I, O, 2, 1), x=None, dy=None, dx=None)])
def test_backward_takes(no_gpu, more):
    assert passes_the_checks(backward(**more))


@pytest.mark.parametrize("shape", [(1, 64, 128, 1, 1), (257, 1024, 4096, 8, 4), (16384, 2560, 10240, 8, 4), (0, 64, 128, 1, 1)])
def test_workspace_sizes(shape):
    for bwd in (False, True):
        base, peak = osdp.osdp_split_linear_workspace_bytes(*shape, bwd)
        total, peak2 = osdp.osdp_split_linear_epilogue_workspace_bytes(*shape, bwd)
        assert peak2 == peak and total >= base and (bwd or total == base)
        assert total - base < 256 + 4 * 1024 * shape[2]
    # one byte less than what is asked for is refused before anything runs
    total, _ = osdp.osdp_split_linear_epilogue_workspace_bytes(*shape, True)
    assert backward(shape=shape, ws_bytes=total - 1, x=P, dy=1 << 44, dx=1 << 45, z=1 << 46, dz=1 << 47, dbias=1 << 48, ldz=shape[2], lddz=shape[2],
                    lddy=shape[2]) in (WORKSPACE, INVALID, UNSUPPORTED)


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    X, Y, w = torch.zeros(4, 64).bfloat16(), torch.zeros(4, 128).bfloat16(), [torch.zeros(64 * 128).bfloat16()]
    ws = torch.zeros(1024, dtype=torch.uint8)
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_split_linear_fwd_epilogue(X, w, Y, 1, ws, epilogue=osdp.Epilogue())
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_split_linear_bwd_epilogue(X, Y, w, X, w, 1, ws, epilogue=osdp.EpilogueGrad())
    q = torch.zeros(4, 2, 64).bfloat16()
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_qk_norm_rope_fwd(q, q, q, q)
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_qk_norm_rope_bwd(q, q, q, q, q, q, None, None, None)


# ---- norms and rotation of queries and keys -----------------------------------------------------------------------
D, HQ, HK = 64, 4, 2
ROW = (HQ + 2 * HK) * D


def desc(**more):
    d = B.osdp_qk(T, HQ, HK, D, D, 0, 1, B.OSDP_BF16, 0, 1e-6, 20 * P, 21 * P, 22 * P, 23 * P)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def heads(p, ld=ROW, hs=D):
    return ctypes.byref(B.osdp_heads(p, ld, hs))


def qk_forward(q=None, k=None, q_out=None, k_out=None, d=True, **more):
    return osdp.lib.osdp_qk_norm_rope_fwd(ctypes.byref(desc(**more)) if d else None, q or heads(P), k or heads(P + 2 * HQ * D),
                                          q_out or heads(2 * P, HQ * D), k_out or heads(3 * P, HK * D), None)


def qk_backward(dq_out=None, dk_out=None, dq=None, dk=None, wq=24 * P, wk=25 * P, ws=26 * P, ws_bytes=1 << 30, **more):
    return osdp.lib.osdp_qk_norm_rope_bwd(ctypes.byref(desc(**more)), heads(P), heads(P + 2 * HQ * D), dq_out or heads(2 * P, HQ * D),
                                          dk_out or heads(3 * P, HK * D), dq or heads(4 * P), dk or heads(4 * P + 2 * HQ * D), wq, wk, ws,
                                          ws_bytes, None)


COMMON = [
    (dict(T=-1), INVALID), (dict(q_heads=-1), INVALID), (dict(D=0), INVALID), (dict(rotary=-16), INVALID), (dict(rotary=80), INVALID),
    (dict(interleaved=2), INVALID), (dict(norm=2), INVALID), (dict(reserved=1), INVALID), (dict(weight_type=2), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(eps=-1.0), INVALID), (dict(norm=0), INVALID), (dict(freqs=None), INVALID),
    (dict(D=68), UNSUPPORTED), (dict(D=520), UNSUPPORTED), (dict(rotary=24), UNSUPPORTED), (dict(rotary=20, interleaved=1), UNSUPPORTED),
    (dict(T=1 << 31), UNSUPPORTED), (dict(k_heads=65536), UNSUPPORTED), (dict(q_weight=22 * P + 8), UNSUPPORTED), (dict(positions=20 * P + 4), UNSUPPORTED),
    (dict(freqs=21 * P + 4), UNSUPPORTED)]


@pytest.mark.parametrize("more,status", COMMON + [
    (dict(d=False), INVALID), (dict(q=heads(None)), INVALID), (dict(k_out=heads(None)), INVALID), (dict(q=heads(P, -8)), INVALID),
    (dict(q=heads(P, ROW + 4)), UNSUPPORTED), (dict(k=heads(P + 2 * HQ * D, ROW, D + 4)), UNSUPPORTED), (dict(q=heads(P + 8)), UNSUPPORTED),
    (dict(q_out=heads(2 * P, HQ * D, D - 8)), INVALID), (dict(q_out=heads(2 * P, (HQ - 1) * D)), INVALID), (dict(k_out=heads(3 * P, 0)), INVALID),
    (dict(q_out=heads(P + 16)), INVALID), (dict(q_out=heads(P, ROW + 8)), INVALID), (dict(k_out=heads(P)), INVALID), (dict(k_out=heads(2 * P, HQ * D)), INVALID),
    (dict(q_out=heads(P + 2 * HQ * D)), INVALID), (dict(k_out=heads(P + 2 * (HQ - 1) * D)), INVALID)])
def test_qk_forward_refuses(more, status):
    assert qk_forward(**more) == status
    assert osdp.lib.osdp_last_error()


@pytest.mark.parametrize("more", [
    dict(), dict(q_out=heads(P), k_out=heads(P + 2 * HQ * D)), dict(q_out=heads(2 * P, D, T * D), k_out=heads(3 * P, D, T * D)),
    dict(q=heads(P, ROW, 2 * D), k=heads(P + 2 * D, ROW, 4 * D), q_out=heads(P, ROW, 2 * D), k_out=heads(P + 2 * D, ROW, 4 * D)),
    dict(norm=0, q_weight=None, k_weight=None), dict(rotary=0, freqs=None), dict(positions=None), dict(k_heads=0, k=heads(None), k_out=heads(None)),
    dict(T=0, q=heads(None), k=heads(None), q_out=heads(None), k_out=heads(None))])
def test_qk_forward_takes(no_gpu, more):
    """In place, by head, heads of queries and keys in turn, without norm, rotation, positions, keys, tokens."""
    assert passes_the_checks(qk_forward(**more))


@pytest.mark.parametrize("more,status", COMMON + [
    (dict(norm=0, q_weight=None, k_weight=None), INVALID), (dict(wq=24 * P + 8), UNSUPPORTED), (dict(wk=24 * P), INVALID), (dict(ws=None), INVALID),
    (dict(ws=26 * P + 64), UNSUPPORTED), (dict(ws_bytes=64), WORKSPACE), (dict(dq=heads(4 * P, 0)), INVALID), (dict(dq=heads(P + 16)), INVALID),
    (dict(dk=heads(P)), INVALID), (dict(dk=heads(2 * P, HQ * D)), INVALID), (dict(dk=heads(4 * P)), INVALID), (dict(dq_out=heads(None)), INVALID)])
def test_qk_backward_refuses(more, status):
    assert qk_backward(**more) == status


@pytest.mark.parametrize("more", [
    dict(), dict(dq=heads(P), dk=heads(P + 2 * HQ * D)), dict(dq=heads(2 * P, HQ * D), dk=heads(3 * P, HK * D)), dict(wq=None, wk=None, ws=None, ws_bytes=0),
    dict(wk=None), dict(norm=0, q_weight=None, k_weight=None, wq=None, wk=None)])
def test_qk_backward_takes(no_gpu, more):
    assert passes_the_checks(qk_backward(**more))


def test_qk_workspace_sizes():
    sizes = [osdp.osdp_qk_norm_rope_bwd_workspace_bytes(t, 32, 8, 128) for t in (0, 1, 100, 8192, 1 << 30)]
    assert sizes[0] == 0 and sizes == sorted(sizes) and sizes[-1] <= 1024 * 128 * 4
    for bad in ((-1, 1, 1, 64), (1, -1, 1, 64), (1, 1, 1, 0), (1, 1, 1, 20), (1, 1, 1, 1024), (1 << 31, 1, 1, 64)):
        with pytest.raises(osdp.OsdpError):
            osdp.osdp_qk_norm_rope_bwd_workspace_bytes(*bad)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(B.osdp_epilogue) == 48 and ctypes.sizeof(B.osdp_epilogue_grad) == 48
    assert ctypes.sizeof(B.osdp_qk) == 80 and ctypes.sizeof(B.osdp_heads) == 24


def test_the_short_way_into_the_library_answers_only_what_it_knows():
    """Anything but the common call is left to Python: None, and nothing raised."""
    calls, t = B._calls, torch.zeros(4, 2, 64).bfloat16()
    assert calls.qk() is None and calls.qk(1, 2, 3) is None and calls.linear() is None and calls.linear(*range(13)) is None and calls.linear(*range(15)) is None
    for heads_ in ((t,) * 4, (t,) * 5, (1, 2, 3, 4), ()):
        assert calls.qk(heads_, None, None, None, None, None, None, None, 1e-6, True, False, None) is None
    assert calls.qk((t,) * 4, None, None, None, None, None, None, None, 1, True, False, None) is None
    X, w = torch.zeros(4, 64).bfloat16(), [torch.zeros(64 * 64).bfloat16()]
    ws = torch.zeros(256, dtype=torch.uint8)
    for plan in (None, osdp.Plan([1]), osdp.Plan([]), osdp.Plan([1.5]), osdp.Plan([1] * 100), "plan"):
        assert calls.linear(X, w, X, 1, ws, plan, 0, None, None, 0, None, None, None) is None
    assert calls.linear(X, [], X, 1, ws, None, 0, None, None, 0, None, None, None) is None
    assert calls.linear(X, w * 65, X, 1, ws, None, 0, None, None, 0, None, None, None) is None
    assert calls.linear(X, [None], X, 1 << 80, ws, None, 0, "s", None, 0, None, None, None) is None
    with pytest.raises(TypeError):
        calls.connect(1, 2)


@pytest.mark.parametrize("more", [dict(x=2 * P, ldx=0, ldy=0), dict(x=2 * P + 16, ldx=0, ldy=0), dict(ldx=0), dict(ldy=0), dict(x=2 * P, ldx=-O, ldy=-O),
                                  dict(ldz=0), dict(ld_residual=0), dict(z=2 * P, ldz=0, ldy=0), dict(shape=(T, I, O, 2, 1), x=2 * P, ldx=0, ldy=0, z=None, residual=None)])
def test_forward_refuses_rows_that_lie_on_each_other(more):
    """Leading dimensions of 0 (an expanded tensor's) and below, alone and in two overlapping matrices."""
    assert forward(**more) == INVALID
    assert osdp.lib.osdp_last_error()


@pytest.mark.parametrize("more", [dict(dy=6 * P, lddy=0, lddz=0), dict(lddy=0), dict(ldz=0, lddz=0, z=6 * P), dict(lddz=0), dict(dx=P, lddy=0), dict(lddy=-O)])
def test_backward_refuses_rows_that_lie_on_each_other(more):
    assert backward(**more) == INVALID
    assert osdp.lib.osdp_last_error()


def elements(p, ld, hs, tokens, n, D):
    return {p // 2 + t * ld + h * hs + d for t in range(tokens) for h in range(n) for d in range(D)}


def test_heads_that_share_memory_are_refused_and_others_are_not(no_gpu):
    """Rows of one length, heads within a row or rows within a head, strides with and without a common divisor: every overlap that
    there is, and no other, between the outputs and between an output and the other side's input."""
    rng, seen = random.Random(5), {True: 0, False: 0}
    for _ in range(6000):
        t, n = rng.choice([1, 2, 3, 5]), [rng.choice([1, 1, 2, 3, 4]) for _ in range(2)]
        d = rng.choice([8, 16, 24])
        sides, row = [], 8 * rng.randint(d // 8, 14)
        for i in range(2):
            written = i == 0 or rng.random() < 0.5
            hs = 8 * rng.randint(d // 8 if written else 0, 8) if rng.random() < 0.5 else rng.choice([row * t, row * t + 8, 2 * row * t, row * (t + 1) - 8])
            sides.append((4 * P + 16 * rng.randint(0, 60) * i, row, hs, written))
        (a, _, hs_a, _), (b, _, hs_b, b_written) = sides
        itself = lambda hs, heads: not (heads == 1 or t == 1 or row >= (heads - 1) * hs + d or hs >= (t - 1) * row + d)  # noqa: E731
        if itself(hs_a, n[0]) or b_written and itself(hs_b, n[1]) or n[0] > 1 and hs_a < d:
            continue
        want = bool(elements(a, row, hs_a, t, n[0], d) & elements(b, row, hs_b, t, n[1], d))
        size = dict(T=t, q_heads=n[0], k_heads=n[1], D=d, rotary=0, freqs=None)
        apart = dict(q=heads(P, 64 * d, d), q_out=heads(a, row, hs_a))
        if b_written:
            status = qk_forward(**size, **apart, k=heads(2 * P, 64 * d, d), k_out=heads(b, row, hs_b))
        else:
            status = qk_forward(**size, **apart, k=heads(b, row, hs_b), k_out=heads(2 * P, 64 * d, d))
        assert passes_the_checks(status) != want, (size, sides, osdp.lib.osdp_last_error())
        seen[want] += 1
    assert min(seen.values()) > 500


@pytest.mark.parametrize("more", [
    # head 0 of the keys' token 50 is head 1 of the queries' token 0
    dict(T=100, q_heads=2, k_heads=2, q_out=heads(4 * P, 256, 25728), k_out=heads(4 * P + 2 * 12928, 256, 25728)),
    dict(q_out=heads(4 * P, 2 ** 59)), dict(q=heads(P, ROW, 2 ** 60))])
def test_qk_forward_refuses_heads_in_each_other(more):
    assert qk_forward(**more) == INVALID


@pytest.mark.parametrize("more", [
    dict(q_heads=2, k_heads=2, q_out=heads(4 * P, D, 2 * T * D), k_out=heads(4 * P + 2 * T * D, D, 2 * T * D)),   # [heads, 2, tokens, D]
    dict(q_heads=4, k_heads=2, q_out=heads(4 * P, D, 2 * T * D), k_out=heads(4 * P + 2 * T * D, D, 4 * T * D)),
    dict(q_heads=2, k_heads=2, q_out=heads(4 * P, 2 * D, 4 * T * D), k_out=heads(4 * P + 2 * D, 2 * D, 4 * T * D))])  # [heads, .., tokens, 2, D]
def test_qk_forward_takes_heads_in_turn_by_head(no_gpu, more):
    assert passes_the_checks(qk_forward(**more))


@pytest.mark.parametrize("tokens,q_heads,k_heads,D", [(100, 64, 64, 512), (64, 64, 8, 256), (3, 100, 100, 64), (300, 48, 1, 128), (1, 65535, 65535, 8), (1, 32, 8, 128), (767, 64, 1, 512)])
def test_qk_backward_asks_for_no_plane_that_no_token_adds_to(tokens, q_heads, k_heads, D):
    """A workgroup walks all heads of its tokens: each side has a plane of D sums for each token tile at most, which holds one token or more,
    and both sides together have 768."""
    planes = osdp.osdp_qk_norm_rope_bwd_workspace_bytes(tokens, q_heads, k_heads, D) // (4 * D)
    assert 2 <= planes <= min(2 * tokens, 768)


def test_qk_backward_gives_both_sides_workgroups():
    """With more token tiles than workgroups that run at once: 768 in all, and for one side without heads too."""
    for q_heads, k_heads in ((64, 1), (1, 64), (8, 8), (64, 0), (0, 1), (65535, 1)):
        assert osdp.osdp_qk_norm_rope_bwd_workspace_bytes(1 << 20, q_heads, k_heads, 512) == 768 * 512 * 4


@pytest.mark.parametrize("weight_type,size", [(B.OSDP_BF16, 2), (B.OSDP_F32, 4)])
def test_qk_backward_refuses_weight_gradients_in_each_other(weight_type, size):
    for off in (0, 16, D * size - 16):
        assert qk_backward(weight_type=weight_type, wk=24 * P + off) == INVALID
        assert qk_backward(weight_type=weight_type, wq=24 * P + off, wk=24 * P) == INVALID


@pytest.mark.parametrize("weight_type,size", [(B.OSDP_BF16, 2), (B.OSDP_F32, 4)])
def test_qk_backward_takes_weight_gradients_side_by_side(no_gpu, weight_type, size):
    assert passes_the_checks(qk_backward(weight_type=weight_type, wk=24 * P + D * size))
