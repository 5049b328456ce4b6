"""Norms of queries and keys and their rotation by position, and the pass back, against the formulas in 64 bits.

Tolerances, in units of the head's largest magnitude m where terms of a pair can cancel.  Forward: a squared sum of D <= 512 products
in fp32 is off by at most (D / 16 + 6) 2^-24 of itself (16 in a lane, then pairs of lanes), half of that in the root; root, reciprocal, weight, cosine and sine,
products and sum add 8 roundings of 2^-24 and 2^-20 from the hardware's cosine and sine: under 2^-18 of the pair's size, at most
sqrt 2 m.  Then half a step of bf16, 2^-8 of the value.  Backward: the same on gradients, and mean(t xh) the same again, times |xh| <= sqrt D:
2^-15 of the largest |r t|, D^1/2 2^-19 of it for the last term.  dg: T H terms off by 2^-17 each (of |dn xh| of the pair), and the sum in fp32."""
from __future__ import annotations

import pytest
import torch

import epilogue_reference as R
import paper_2209_13258_amd as osdp

pytestmark = pytest.mark.gpu


def rand(*shape, std=1.0, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(hash((shape, seed)) % (1 << 31))
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def some_freqs(rotary, base=10000.0):
    return base ** (-2.0 * torch.arange(rotary // 2, dtype=torch.float64, device="cuda") / rotary) if rotary else None


def close(got, want, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got - want).abs() - bound
    assert off.max().item() <= 0, f"{what}: {int((off > 0).sum())} values beyond the bound, by up to {off.max().item():.3e}"


def check_forward(got, x, pos, freqs, weight, norm=True, interleaved=False, eps=1e-6):
    want = R.qk(x.double(), pos, freqs, weight, eps, norm, interleaved)
    close(got, want, 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True) * 1.5, "heads")


def check_backward(dx, dg, x, dy, pos, freqs, weight, norm=True, interleaved=False, eps=1e-6):
    want, want_g = R.qk_back(x.double(), dy.double(), pos, freqs, weight, eps, norm, interleaved)
    D, rt = x.shape[-1], dy.double().abs()
    if norm:
        r = 1 / (x.double().square().mean(-1, keepdim=True) + eps).sqrt()
        rt = rt * r * (1.0 if weight is None else weight.double().abs().max())
    scale = rt.amax(-1, keepdim=True) * (2.0 ** -15 + D ** 0.5 * 2.0 ** -19)
    close(dx, want, 2.0 ** -8 * want.abs() + 2 * scale, "dx")
    if dg is not None:
        xh = x.double() * r
        terms = (dy.double().abs().amax(-1, keepdim=True) * 2 * xh.abs()).sum((0, 1))
        n = x.shape[0] * x.shape[1]
        half = 2.0 ** -8 if dg.dtype == torch.bfloat16 else 2.0 ** -24
        close(dg, want_g, terms * (2.0 ** -17 + min(n, 4096) * 2.0 ** -24) + half * (want_g.abs() + terms * 2.0 ** -16), "dg")


def forward(q, k, q_out=None, k_out=None, **how):
    q_out = torch.full_like(q, float("nan"), memory_format=torch.contiguous_format) if q_out is None else q_out
    k_out = torch.full_like(k, float("nan"), memory_format=torch.contiguous_format) if k_out is None else k_out
    osdp.osdp_qk_norm_rope_fwd(q, k, q_out, k_out, **how)
    return q_out, k_out


def workspace(T, HQ, HK, D):
    return torch.full((max(osdp.osdp_qk_norm_rope_bwd_workspace_bytes(T, HQ, HK, D), 256),), 0xFF, dtype=torch.uint8, device="cuda")


def backward(q, k, dq_out, dk_out, dq=None, dk=None, dtype=torch.bfloat16, weights=True, stream=None, **how):
    T, HQ, D = q.shape
    dq = torch.full((T, HQ, D), float("nan"), dtype=torch.bfloat16, device="cuda") if dq is None else dq
    dk = torch.full((T, k.shape[1], D), float("nan"), dtype=torch.bfloat16, device="cuda") if dk is None else dk
    dg = [torch.full((D,), float("nan"), dtype=dtype, device="cuda") if weights else None for _ in range(2)]
    osdp.osdp_qk_norm_rope_bwd(q, k, dq_out, dk_out, dq, dk, *dg, workspace(T, HQ, k.shape[1], D) if weights else None, stream=stream, **how)
    return dq, dk, *dg


# (T, query heads, key heads, D, rotary in halves, rotary interleaved)
SHAPES = [(1, 1, 1, 8, 0, 8), (1, 32, 8, 128, 128, 128), (2, 3, 1, 16, 16, 8), (5, 4, 4, 24, 16, 24), (17, 6, 2, 32, 32, 8), (3, 64, 8, 40, 32, 40), (100, 5, 5, 64, 64, 64),
          (1001, 32, 32, 80, 32, 80), (33, 7, 1, 96, 96, 48), (700, 1, 8, 112, 96, 104), (2048, 32, 8, 128, 128, 64), (64, 2, 3, 136, 128, 136), (9, 16, 16, 256, 64, 256),
          (40, 3, 3, 264, 256, 264), (6, 4, 2, 512, 512, 512), (8192, 8, 2, 64, 64, 64), (300, 100, 12, 64, 32, 16)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forward_and_backward(shape, interleaved, dtype):
    T, HQ, HK, D, half, inter = shape
    rotary = inter if interleaved else half
    rows = rand(T, (HQ + 2 * HK) * D)
    q, k = rows[:, :HQ * D].unflatten(1, (HQ, D)), rows[:, HQ * D:(HQ + HK) * D].unflatten(1, (HK, D))
    w = [rand(D, std=0.3, seed=s, dtype=torch.float32).add_(1).to(dtype) for s in (1, 2)]
    pos, freqs = torch.randint(0, 100000, (T,), device="cuda"), some_freqs(rotary)
    how = dict(positions=pos, freqs=freqs, q_weight=w[0], k_weight=w[1], interleaved=interleaved)
    q_out, k_out = forward(q, k, **how)
    check_forward(q_out, q, pos, freqs, w[0], interleaved=interleaved)
    check_forward(k_out, k, pos, freqs, w[1], interleaved=interleaved)
    dq_out, dk_out = rand(T, HQ, D, seed=3), rand(T, HK, D, seed=4)
    dq, dk, dgq, dgk = backward(q, k, dq_out, dk_out, dtype=dtype, **how)
    check_backward(dq, dgq, q, dq_out, pos, freqs, w[0], interleaved=interleaved)
    check_backward(dk, dgk, k, dk_out, pos, freqs, w[1], interleaved=interleaved)
    # without the weights' gradients the others are the same bits
    again = backward(q, k, dq_out, dk_out, weights=False, **how)
    assert torch.equal(again[0], dq) and torch.equal(again[1], dk)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rotary", [0, 64])
@pytest.mark.parametrize("sides", [(4, 0), (0, 3), (4, 3), (0, 0)])
def test_parts_can_be_left_out(norm, rotary, sides):
    """No norm, no weights, no rotation, no positions, no queries, no keys."""
    T, D = 50, 64
    q, k = rand(T, sides[0], D), rand(T, sides[1], D, seed=1)
    pos, freqs = torch.arange(T, device="cuda"), some_freqs(rotary)
    for x, y in zip((q, k), forward(q, k, freqs=freqs, norm=norm)):
        if x.numel():
            check_forward(y, x, pos, freqs, None, norm)
    dy = [rand(T, n, D, seed=2) for n in sides]
    out = backward(q, k, *dy, freqs=freqs, norm=norm, weights=norm, dtype=torch.float32)
    for i, x in enumerate((q, k)):
        if x.numel():
            check_backward(out[i], out[2 + i], x, dy[i], pos, freqs, None, norm)
        elif norm:
            assert (out[2 + i] == 0).all()


def test_no_tokens():
    q = rand(0, 4, 64)
    forward(q, q)
    out = backward(q, q, q, q, dtype=torch.float32)
    assert (out[2] == 0).all() and (out[3] == 0).all()


@pytest.mark.parametrize("T", [3, 2000])
def test_layouts(T):
    """Heads by token, by head, queries and keys in turn, with gaps; in place; what lies between them stays as it was."""
    H, D = 6, 80
    base = rand(T, H, D), rand(T, H, D, seed=1)
    pos = torch.randint(0, 5000, (T,), device="cuda")
    how = dict(positions=pos, freqs=some_freqs(80), q_weight=rand(D, seed=2), k_weight=rand(D, seed=3))
    want = forward(*base, **how)
    dy = rand(T, H, D, seed=4), rand(T, H, D, seed=5)
    want_back = backward(*base, *dy, **how)

    def by_head():
        return torch.full((2, H, T, D), 7.0, dtype=torch.bfloat16, device="cuda"), lambda b: (b[0].transpose(0, 1), b[1].transpose(0, 1))

    def in_turn():
        return torch.full((T, H, 3, D), 7.0, dtype=torch.bfloat16, device="cuda"), lambda b: (b[:, :, 0], b[:, :, 1])

    def gaps():
        return torch.full((T, 2 * H + 1, D + 16), 7.0, dtype=torch.bfloat16, device="cuda"), lambda b: (b[:, :H, 8:8 + D], b[:, H + 1:, 8:8 + D])

    for layout in (by_head, in_turn, gaps):
        buf, views = layout()
        out = views(buf)
        forward(*base, *out, **how)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        for v in out:
            v.fill_(7.0)
        assert (buf == 7.0).all()                       # nothing beside the heads was written
        for v, x in zip(out, base):
            v.copy_(x)
        forward(*out, *out, **how)                      # in place
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        for v, x in zip(out, base):
            v.copy_(x)
        grads = backward(*out, *dy, *out, **how)        # dq in the place of q
        assert all(torch.equal(a, b) for a, b in zip(grads, want_back))
        for v, x in zip(out, dy):
            v.copy_(x)
        grads = backward(*base, *out, *out, **how)      # dq in the place of dq_out
        assert all(torch.equal(a, b) for a, b in zip(grads, want_back))


@pytest.mark.parametrize("T,H,D", [(1, 4, 64), (37, 5, 64), (1000, 32, 128), (64, 1, 24)])
def test_rows_of_padding_are_left_alone(T, H, D):
    """Negative positions, the rows full of NaN: outputs untouched, nothing added to the weights' gradients."""
    q, k, dy = rand(T, H, D), rand(T, 2, D, seed=1), rand(T, H, D, seed=2)
    dk_out = rand(T, 2, D, seed=3)
    pos = torch.randint(0, 1000, (T,), device="cuda")
    pad = torch.rand(T, device="cuda") < 0.4
    pad[0] = True
    pos[pad] = torch.where(torch.rand(int(pad.sum()), device="cuda") < 0.5, -1, -(1 << 62))
    for t in (q, k, dy, dk_out):
        t[pad] = float("nan")
    how = dict(positions=pos, freqs=some_freqs(16), q_weight=rand(D, seed=4, dtype=torch.float32), k_weight=rand(D, seed=5, dtype=torch.float32))
    out = forward(q, k, torch.full_like(q, 3.0), torch.full_like(k, 3.0), **how)
    back = backward(q, k, dy, dk_out, torch.full_like(q, 3.0), torch.full_like(k, 3.0), dtype=torch.float32, **how) if not pad.all() else None
    live = ~pad
    for i, (x, g, w) in enumerate(((q, dy, how["q_weight"]), (k, dk_out, how["k_weight"]))):
        assert (out[i][pad] == 3.0).all()
        if live.any():
            check_forward(out[i][live], x[live], pos[live], how["freqs"], w)
            assert (back[i][pad] == 3.0).all()
            check_backward(back[i][live], back[2 + i], x[live], g[live], pos[live], how["freqs"], w)


def test_a_batch_of_padding_gives_zero_gradients():
    q = torch.full((5, 3, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    pos = torch.full((5,), -1, dtype=torch.int64, device="cuda")
    out = backward(q, q, q, q, positions=pos, freqs=some_freqs(64), dtype=torch.float32)
    assert (out[2] == 0).all() and (out[3] == 0).all()


@pytest.mark.parametrize("far", [0, 1 << 17, (1 << 31) - 1, 1 << 40])
def test_far_positions(far):
    """The angle of position 2^40 times 1 radian, to less than 2^-12 of a turn even there (2^40 / 2 pi has 38 bits of 53 before the point; the reference,
    in 64 bits too, is as far off)."""
    q = rand(64, 4, 128)
    pos, freqs = far + torch.arange(64, device="cuda"), some_freqs(128)
    got, _ = forward(q, q[:, :1], positions=pos, freqs=freqs)
    want = R.qk(q.double(), pos, freqs, None, 1e-6, True, False)
    slack = 2 * 6.2832 * far * 2.0 ** -52  # (radians that either product may be off by)
    close(got, want, 2.0 ** -8 * want.abs() + (2.0 ** -18 * 1.5 + slack) * want.abs().amax(-1, keepdim=True), "heads")


@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -60, 2.0 ** -10, 2.0 ** 20, 2.0 ** 50, 2.0 ** 66, 2.0 ** 120])
@pytest.mark.parametrize("D", [64, 512])
def test_sizes_of_heads(size, D):
    """Heads whose squares leave the range of fp32 upwards, and heads far below eps."""
    q, dy = rand(30, 3, D, std=size), rand(30, 3, D, seed=1)
    w = rand(D, std=0.2, seed=2, dtype=torch.float32).add_(1)
    how = dict(freqs=some_freqs(D), q_weight=w, k_weight=w, positions=torch.arange(30, device="cuda"))
    out = forward(q, q, **how)[0]
    want = R.qk(q.double(), how["positions"], how["freqs"], w, 1e-6, True, False)
    tiny = 2.0 ** -133  # (half a step of the smallest bf16 numbers)
    close(out, want, 2.0 ** -8 * want.abs() + 2.0 ** -18 * 1.5 * want.abs().amax(-1, keepdim=True) + tiny, "heads")
    dx, _, dg, _ = backward(q, q, dy, dy, dtype=torch.float32, **how)
    want, want_g = R.qk_back(q.double(), dy.double(), how["positions"], how["freqs"], w, 1e-6, True, False)
    rms = want.square().mean().sqrt()
    assert ((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * rms + tiny).all()
    assert ((dg.double() - want_g).abs() <= 2.0 ** -10 * want_g.square().mean().sqrt() + 2.0 ** -126).all()


def test_zeros_infinities_and_nan_stay_in_their_heads():
    q = rand(8, 4, 64)
    clean = q.clone()
    q[1, 2] = 0
    q[3, 1, 5] = float("nan")
    q[5, 0, 7] = float("inf")
    out, _ = forward(q, q[:, :1], freqs=some_freqs(64))
    ref, _ = forward(clean, clean[:, :1], freqs=some_freqs(64))
    assert (out[1, 2] == 0).all() and torch.isnan(out[3, 1]).all() and torch.isnan(out[5, 0, 7])
    same = torch.ones(8, 4, dtype=torch.bool, device="cuda")
    same[1, 2] = same[3, 1] = same[5, 0] = False
    assert torch.equal(out[same], ref[same])


@pytest.mark.parametrize("interleaved", [False, True])
def test_what_is_not_turned_does_not_see_its_neighbours(interleaved):
    """Without a norm, elements behind the rotated ones are copied, whatever lies beside them."""
    q = rand(6, 2, 64)
    q[..., 40] = float("inf")
    q[..., 63] = float("nan")
    out, _ = forward(q, q, freqs=some_freqs(16), norm=False, interleaved=interleaved, positions=torch.arange(6, device="cuda"))
    assert torch.equal(out[..., 16:].view(torch.int16), q[..., 16:].view(torch.int16)) and torch.isfinite(out[..., :16]).all()
    back = backward(q, q, q, q, freqs=some_freqs(16), norm=False, interleaved=interleaved, weights=False, positions=torch.arange(6, device="cuda"))[0]
    assert torch.equal(back[..., 16:].view(torch.int16), q[..., 16:].view(torch.int16)) and torch.isfinite(back[..., :16]).all()


def test_turned_back_is_what_was_turned():
    """Without a norm the pass back is the inverse rotation: the gradient of half the squared size is the input itself."""
    q = rand(100, 4, 128)
    how = dict(freqs=some_freqs(128), norm=False, positions=torch.randint(0, 1 << 20, (100,), device="cuda"))
    there, _ = forward(q, q, **how)
    back = backward(q, q, there, there, weights=False, **how)[0]
    m = q.double().abs().amax(-1, keepdim=True)
    assert ((back.double() - q.double()).abs() <= 2.0 ** -8 * q.double().abs() + (2.0 ** -8 * 2 + 2.0 ** -17) * m).all()


def test_offsets_beyond_32_bits():
    T, ld = 9000, 1 << 18
    wide = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)
    q, k, dq = (wide[:, 1024 * i:1024 * i + 512].unflatten(1, (8, 64)) for i in range(3))
    q.copy_(rand(T, 8, 64))
    k.copy_(rand(T, 8, 64, seed=1))
    how = dict(freqs=some_freqs(64), positions=torch.arange(T, device="cuda"), q_weight=rand(64, seed=2), k_weight=rand(64, seed=3))
    near_q, near_k = q.contiguous(), k.contiguous()
    dy = rand(T, 8, 64, seed=4)
    want, want_back = forward(near_q, near_k, **how), backward(near_q, near_k, dy, dy, **how)
    back = backward(q, k, dy, dy, dq, None, **how)
    assert all(torch.equal(a, b) for a, b in zip(back, want_back))
    forward(q, k, q, k, **how)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("T", [1, 900])
def test_a_captured_graph_replays_on_other_inputs(T):
    HQ, HK, D = 8, 2, 64
    q, k, dy, dk_out = rand(T, HQ, D), rand(T, HK, D, seed=1), rand(T, HQ, D, seed=2), rand(T, HK, D, seed=3)
    pos, freqs, w = torch.arange(T, device="cuda"), some_freqs(D), rand(D, seed=4)
    outs = [torch.empty_like(t) for t in (q, k, q, k, w, w)]
    ws = workspace(T, HQ, HK, D)

    def run(stream):
        how = dict(positions=pos, freqs=freqs, q_weight=w, k_weight=w, stream=stream)
        osdp.osdp_qk_norm_rope_fwd(q, k, outs[0], outs[1], **how)
        osdp.osdp_qk_norm_rope_bwd(q, k, dy, dk_out, *outs[2:], ws, **how)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    run(stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(stream)
    for seed in range(4):
        q.copy_(rand(T, HQ, D, seed=70 + seed))
        pos.add_(1000)
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        run(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), seed


def test_the_same_inputs_give_the_same_bits():
    q, k, dy, dk = rand(3000, 16, 64), rand(3000, 4, 64, seed=1), rand(3000, 16, 64, seed=2), rand(3000, 4, 64, seed=3)
    runs = [backward(q, k, dy, dk, freqs=some_freqs(64), dtype=torch.float32) for _ in range(5)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


def test_the_binding_refuses_what_does_not_fit():
    q, k, w = rand(5, 4, 64), rand(5, 2, 64, seed=1), rand(64)
    pos, freqs = torch.arange(5, device="cuda"), some_freqs(64)
    wrong = [dict(positions=pos.int()), dict(positions=pos[:4]), dict(positions=pos.cpu()), dict(freqs=freqs.float()), dict(freqs=freqs.cpu()),
             dict(freqs=some_freqs(128)), dict(freqs=freqs[::2]), dict(q_weight=w[:32]), dict(q_weight=w.half()), dict(q_weight=w, k_weight=w.float()),
             dict(q_weight=w, norm=False), dict(eps=0.0), dict(positions=torch.arange(10, device="cuda")[::2])]
    for how in wrong:
        with pytest.raises(osdp.OsdpError):
            forward(q, k, **how)
    for a, b, c, d in ((q.float(), k, q, k), (q, k[:4], q, k), (q, k[..., :32], q, k), (q, k, q[:, :3], k), (q, k, q, k.float()), (q, k, q, q[:, :2]),
                       (q.transpose(1, 2).contiguous().transpose(1, 2), k, torch.empty_like(q), k), (q, k, q[:1].expand(5, 4, 64), k), (q, k, q.cpu(), k)):
        with pytest.raises(osdp.OsdpError):
            osdp.osdp_qk_norm_rope_fwd(a, b, c, d)
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_qk_norm_rope_bwd(q, k, q, k, torch.empty_like(q), torch.empty_like(k), w.clone(), w.float(), workspace(5, 4, 2, 64), q_weight=w, k_weight=w)
    with pytest.raises(osdp.OsdpError):
        osdp.osdp_qk_norm_rope_bwd(q, k, q, k, torch.empty_like(q), torch.empty_like(k), w.clone(), None, torch.empty(64, dtype=torch.uint8, device="cuda"), q_weight=w)


@pytest.mark.parametrize("eps", [1e-12, 1e8, 1e18, 1e20, 1e30])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 20, 2.0 ** 28, 2.0 ** 31, 2.0 ** 50, 2.0 ** 66])
def test_any_eps_beside_any_size_of_heads(size, eps):
    """eps counts however large the squares beside it are.  Bounds as for other sizes of heads: 30 tokens of 3 heads, terms of dg off
    by 2^-17 each, dx by (2^-15 + 64^1/2 2^-19) of the largest |r t|, some four times the root mean square."""
    q, dy = rand(30, 3, 64, std=size), rand(30, 3, 64, seed=1)
    w = rand(64, std=0.2, seed=2, dtype=torch.float32).add_(1)
    how = dict(freqs=some_freqs(64), q_weight=w, k_weight=w, positions=torch.arange(30, device="cuda"), eps=eps)
    out = forward(q, q, **how)[0]
    check_forward(out, q, how["positions"], how["freqs"], w, eps=eps)
    dx, _, dg, _ = backward(q, q, dy, dy, dtype=torch.float32, **how)
    want, want_g = R.qk_back(q.double(), dy.double(), how["positions"], how["freqs"], w, eps, True, False)
    assert ((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * want.square().mean().sqrt()).all()
    assert ((dg.double() - want_g).abs() <= 2.0 ** -10 * want_g.square().mean().sqrt()).all()


# (T, query heads, key heads, D): one token tile to a workgroup and many, one head group and many
@pytest.mark.parametrize("shape", [(100, 64, 64, 512), (700, 64, 3, 256), (2048, 32, 8, 128), (3000, 16, 4, 64), (5000, 8, 8, 128), (8192, 8, 2, 64), (20000, 3, 1, 80)], ids=str)
def test_no_term_of_the_weights_gradients_is_lost_or_counted_twice(shape):
    """Heads and gradients of +-1: the root mean square is 1, and without rotation dg is a sum of ones of both signs, up to 2^16 of them.
    The factor (its root off by 2^-23, the mean over a D that is no power of two and eps of 1e-12 by 2^-24 each) and its product with a
    gradient move the sum by less than 2^16 2^-21; fewer than 100 additions one after another (a lane's own terms, a workgroup's lane
    groups, the workgroups) by 100 * 2^-24 * 2^16: less than 0.43 in all.  One term more or less moves every element by 1."""
    T, HQ, HK, D = shape
    g = torch.Generator(device="cuda").manual_seed(T)
    sides = []
    for heads in (HQ, HK):
        x = torch.randint(0, 2, (T, heads, D), device="cuda", generator=g).mul_(2).sub_(1).bfloat16()
        sides.append((x, torch.randint(0, 2, (T, heads, D), device="cuda", generator=g).mul_(2).sub_(1).bfloat16()))
    (q, dq_out), (k, dk_out) = sides
    out = backward(q, k, dq_out, dk_out, dtype=torch.float32, eps=1e-12)
    for i, (x, dy) in enumerate(sides):
        want = (x.double() * dy.double()).sum((0, 1))
        assert (out[2 + i].double() - want).abs().max() < 0.43, i


@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("parts", ["all", "no positions", "no rotation", "no weights", "no norm", "no keys"])
def test_both_ways_into_the_library_hand_over_the_same(monkeypatch, T, parts):
    """Tensors are looked at in C, or in Python where that gives no answer: the same bits."""
    HQ, HK, D = 6, 0 if parts == "no keys" else 2, 64
    rows, given = rand(T, (HQ + 2 * HK) * D + 16), []
    q, k = rows[:, :HQ * D].unflatten(1, (HQ, D)), rows[:, HQ * D:(HQ + HK) * D].unflatten(1, (HK, D))
    w = rand(D, seed=1, dtype=torch.float32) if parts not in ("no weights", "no norm") else None
    how = dict(positions=None if parts == "no positions" else torch.randint(0, 1000, (T,), device="cuda"), freqs=None if parts == "no rotation" else some_freqs(32),
               q_weight=w, k_weight=w, eps=1e-5, norm=parts != "no norm", interleaved=parts == "all")
    dy = rand(T, HQ, D, seed=2), rand(T, HK, D, seed=3)
    for way in ("C", "Python"):
        if way == "Python":
            monkeypatch.setattr(osdp.binding, "_calls", type("OnlyPython", (), {"qk": staticmethod(lambda *a: None)}))
        out = [*forward(q, k, **how), *backward(q, k, *dy, dtype=torch.float32, weights=parts != "no norm", **how)]
        given.append([t for t in out if t is not None])
    assert len(given[0]) == len(given[1]) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*given))
