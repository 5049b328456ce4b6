"""AdamW over shards and the operator in 8-bit integers: sizes, layouts and refusals, which need no GPU."""
import ctypes

import pytest

import paper_2209_13258_amd as osdp
from paper_2209_13258_amd import binding as B

P = 1 << 20  # an address that is aligned and that nothing here follows


def tensor(n=1000, **more):
    t = B.osdp_adamw_tensor(n, P, P, P, P, P, P, 0.1)
    for k, v in more.items():
        setattr(t, k, v)
    return t


def options(**more):
    o = B.osdp_adamw_options(1e-3, 0.9, 0.999, 1e-8, 1, 0, 0.0, None, None, None, B.OSDP_BF16, B.OSDP_BF16, 32, 0)
    for k, v in more.items():
        setattr(o, k, v)
    return o


def step(tensors, o):
    arr = (B.osdp_adamw_tensor * max(len(tensors), 1))(*tensors)
    return osdp.lib.osdp_adamw_step(arr, len(tensors), ctypes.byref(o) if o is not None else None, None)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(B.osdp_adamw_tensor) == 64
    assert ctypes.sizeof(B.osdp_adamw_options) == 96


@pytest.mark.parametrize("more", [
    dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5),
    dict(beta2=float("nan")), dict(eps=0.0), dict(eps=1e-13), dict(eps=float("nan")), dict(eps=float("inf")), dict(step=0),
    dict(step=-3), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(max_norm=1.0), dict(grad_type=2), dict(param_type=7),
    dict(param_type=B.OSDP_F32), dict(state_bits=16), dict(state_bits=0)])
def test_step_refuses_options(more):
    assert step([tensor()], options(**more)) == B.OSDP_ERR_INVALID_ARG
    assert osdp.lib.osdp_last_error()


@pytest.mark.parametrize("more,bits,status", [
    (dict(n=-1), 32, B.OSDP_ERR_INVALID_ARG), (dict(n=1 << 40), 32, B.OSDP_ERR_INVALID_ARG),
    (dict(grad=None), 32, B.OSDP_ERR_INVALID_ARG), (dict(param=None), 32, B.OSDP_ERR_INVALID_ARG),
    (dict(m=None), 32, B.OSDP_ERR_INVALID_ARG), (dict(v=None), 32, B.OSDP_ERR_INVALID_ARG),
    (dict(exps=None), 8, B.OSDP_ERR_INVALID_ARG), (dict(weight_decay=-0.5), 32, B.OSDP_ERR_INVALID_ARG),
    (dict(weight_decay=float("nan")), 32, B.OSDP_ERR_INVALID_ARG), (dict(grad=P + 1), 32, B.OSDP_ERR_UNSUPPORTED),
    (dict(param=P + 1), 32, B.OSDP_ERR_UNSUPPORTED), (dict(master=P + 2), 32, B.OSDP_ERR_UNSUPPORTED),
    (dict(m=P + 2), 32, B.OSDP_ERR_UNSUPPORTED), (dict(v=P + 1), 32, B.OSDP_ERR_UNSUPPORTED), (dict(exps=P + 1), 8, B.OSDP_ERR_UNSUPPORTED)])
def test_step_refuses_tensors(more, bits, status):
    assert step([tensor(), tensor(**more)], options(state_bits=bits)) == status


def test_step_refuses_some_masters_and_misplaced_scalars():
    assert step([tensor(), tensor(master=None)], options()) == B.OSDP_ERR_INVALID_ARG
    assert step([tensor()], None) == B.OSDP_ERR_INVALID_ARG
    assert step([tensor()], options(grad_sumsq=P + 4)) == B.OSDP_ERR_UNSUPPORTED
    assert step([tensor()], options(step_device=P + 4)) == B.OSDP_ERR_UNSUPPORTED
    assert step([tensor()], options(lr_device=P + 2)) == B.OSDP_ERR_UNSUPPORTED
    assert osdp.lib.osdp_adamw_step(None, 1, ctypes.byref(options()), None) == B.OSDP_ERR_INVALID_ARG
    assert osdp.lib.osdp_adamw_step(None, -1, ctypes.byref(options()), None) == B.OSDP_ERR_INVALID_ARG


def test_sumsq_sizes_and_refusals():
    def need(lengths):
        arr = (B.osdp_adamw_tensor * len(lengths))(*[tensor(n=n) for n in lengths])
        out = ctypes.c_size_t()
        assert osdp.lib.osdp_adamw_grad_sumsq_workspace_bytes(arr, len(lengths), ctypes.byref(out)) == 0
        return out.value
    assert need([0]) == 0 and need([0, 0, 0]) == 0
    assert 8 <= need([1]) <= need([1 << 20]) <= need([1 << 34])
    assert need([1] * 200) >= 8 * 4 and need([1 << 39] * 3) < 1 << 20
    arr = (B.osdp_adamw_tensor * 1)(tensor())
    call = lambda **k: osdp.lib.osdp_adamw_grad_sumsq(arr, 1, k.get("type", 0), 0, k.get("out", P), k.get("ws", P), k.get("bytes", 1 << 20), None)  # noqa: E731
    assert call(type=5) == B.OSDP_ERR_INVALID_ARG and call(out=None) == B.OSDP_ERR_INVALID_ARG
    assert call(out=P + 4) == B.OSDP_ERR_UNSUPPORTED and call(ws=P + 4) == B.OSDP_ERR_UNSUPPORTED
    assert call(ws=None) == B.OSDP_ERR_INVALID_ARG and call(bytes=0) == B.OSDP_ERR_WORKSPACE
    assert osdp.lib.osdp_adamw_grad_sumsq_workspace_bytes(arr, 1, None) == B.OSDP_ERR_INVALID_ARG


def test_state_values_refusals():
    arr = (B.osdp_adamw_tensor * 1)(tensor())
    one = lambda p: (ctypes.c_void_p * 1)(p)  # noqa: E731
    assert osdp.lib.osdp_adamw_state_values(arr, 1, None, one(P), None) == B.OSDP_ERR_INVALID_ARG
    assert osdp.lib.osdp_adamw_state_values(arr, 1, one(None), one(P), None) == B.OSDP_ERR_INVALID_ARG
    assert osdp.lib.osdp_adamw_state_values(arr, 1, one(P), one(P + 1), None) == B.OSDP_ERR_UNSUPPORTED
    bad = (B.osdp_adamw_tensor * 1)(tensor(exps=None))
    assert osdp.lib.osdp_adamw_state_values(bad, 1, one(P), one(P), None) == B.OSDP_ERR_INVALID_ARG


def i8_fwd(T=4, I=64, O=32, N=2, k=1, X=P, ldx=None, shards=None, scale=P, Y=P, ldy=None, ws=P, ws_bytes=1 << 30):
    shape = B.osdp_shape(T, I, O, N, k)
    tab = (ctypes.c_void_p * max(N, 1))(*(shards or [P] * max(N, 1)))
    return osdp.lib.osdp_split_linear_i8_fwd(ctypes.byref(shape), X, I if ldx is None else ldx, tab, scale, Y,
                                             O if ldy is None else ldy, ws, ws_bytes, None)


@pytest.mark.parametrize("more,status", [
    (dict(I=24), B.OSDP_ERR_UNSUPPORTED), (dict(I=131088, O=8, N=1), B.OSDP_ERR_UNSUPPORTED), (dict(I=0), B.OSDP_ERR_INVALID_ARG),
    (dict(O=12), B.OSDP_ERR_UNSUPPORTED), (dict(O=-8), B.OSDP_ERR_INVALID_ARG), (dict(T=-1), B.OSDP_ERR_INVALID_ARG),
    (dict(T=1 << 31), B.OSDP_ERR_UNSUPPORTED), (dict(N=0), B.OSDP_ERR_INVALID_ARG), (dict(N=65), B.OSDP_ERR_UNSUPPORTED),
    (dict(I=16, O=8, N=16), B.OSDP_ERR_UNSUPPORTED), (dict(k=-1), B.OSDP_ERR_INVALID_ARG), (dict(k=33), B.OSDP_ERR_INVALID_ARG),
    (dict(k=3), B.OSDP_ERR_UNSUPPORTED), (dict(X=None), B.OSDP_ERR_INVALID_ARG), (dict(X=P + 8), B.OSDP_ERR_UNSUPPORTED),
    (dict(ldx=56), B.OSDP_ERR_INVALID_ARG), (dict(ldx=68), B.OSDP_ERR_UNSUPPORTED), (dict(Y=None), B.OSDP_ERR_INVALID_ARG),
    (dict(ldy=24), B.OSDP_ERR_INVALID_ARG), (dict(ldy=36), B.OSDP_ERR_UNSUPPORTED), (dict(shards=[P, None]), B.OSDP_ERR_INVALID_ARG),
    (dict(shards=[P, P + 8]), B.OSDP_ERR_UNSUPPORTED), (dict(scale=None), B.OSDP_ERR_INVALID_ARG), (dict(scale=P + 4), B.OSDP_ERR_UNSUPPORTED),
    (dict(ws=None), B.OSDP_ERR_INVALID_ARG), (dict(ws=P + 16), B.OSDP_ERR_UNSUPPORTED), (dict(ws_bytes=100), B.OSDP_ERR_WORKSPACE)])
def test_i8_forward_refuses(more, status):
    assert i8_fwd(**more) == status
    assert osdp.lib.osdp_last_error()


def test_i8_forward_refuses_outputs_that_overlap_its_tokens():
    """Every workgroup reads the tokens while others store.  Against sets of addresses: rows of one length apart, matrices beside, between, behind and
    in one another."""
    import random
    rng = random.Random(11)
    seen = {True: 0, False: 0}
    for _ in range(3000):
        T, I, O = rng.randrange(1, 5), 16 * rng.randrange(1, 4), 8 * rng.randrange(1, 5)
        ldx = I + 8 * rng.randrange(0, 8)
        ldy = max(ldx, O) if rng.random() < 0.8 else O + 8 * rng.randrange(0, 8)
        d = 8 * rng.randrange(-T * ldy // 8 - 2, T * ldx // 8 + 3)
        cells = lambda at, ld, n: {(at + t * ld + c) for t in range(T) for c in range(0, n, 8)}  # noqa: E731
        meet = bool(cells(0, ldx, I) & cells(d, ldy, O))
        status = i8_fwd(T=T, I=I, O=O, N=1, X=P, ldx=ldx, Y=P + 2 * d, ldy=ldy, shards=[8 * P], ws_bytes=1 << 40)
        if ldx == ldy or T == 1:
            assert (status == B.OSDP_ERR_INVALID_ARG) == meet, (T, I, O, ldx, ldy, d)
        elif meet or status == B.OSDP_ERR_INVALID_ARG:   # rows of different lengths: where the matrices reach into one another at all
            assert status == B.OSDP_ERR_INVALID_ARG and -((T - 1) * ldy + O) < d < (T - 1) * ldx + I, (T, I, O, ldx, ldy, d)
        seen[meet] += 1
    assert min(seen.values()) > 300
    assert i8_fwd(T=0, X=P, Y=P) != B.OSDP_ERR_INVALID_ARG


@pytest.mark.parametrize("T,I,O,N,k", [(1, 16, 8, 1, 0), (500, 2560, 10240, 8, 4), (500, 2560, 10248, 16, 3), (64, 4096, 24, 64, 1),
                                       (65, 4096, 24, 16, 3), (0, 64, 32, 2, 1), (300, 4096, 256, 16, 1), (300, 4096, 1000, 8, 1)])
def test_i8_workspace_follows_the_law(T, I, O, N, k):
    """One byte an element and 1/k of the weight, where slices are gathered; nothing where the shards are read in place.
    What is for the tokens grows with them, and what their number does not decide is a constant."""
    total, peak = osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, k)
    rows = O // N if O % N == 0 else 0
    gathers = T > 64 and rows < 32 or T > 256 and N > 1 and rows % 256 != 0   # (has to, or may)
    assert peak == (I * max((j + 1) * O // max(k, 1) - j * O // max(k, 1) for j in range(max(k, 1))) if gathers else 0)
    tokens = T * (-(-I // 128) * 128) + 4 * T
    assert tokens + peak <= total <= tokens + peak + (16 << 20) + 1024 + 3 * 256
    fewer = [osdp.osdp_split_linear_i8_workspace_bytes(t, I, O, N, k)[0] for t in range(0, T + 1, max(1, T // 50))]
    assert fewer == sorted(fewer) and max(fewer) <= total, "what does for T tokens has to do for fewer"


def test_i8_weights_of_most_channels():
    """A launch counts its threads in 32 bits, so 16 channels to a workgroup of 512 ends at 2^27: a weight of more that is cut within channels is
    gathered for any number of tokens.  Tile numbers and columns behind the last one are 32-bit numbers too."""
    I, O, N = 48, (1 << 27) + 8, 3
    for T in (1, 5, 64, 65):
        assert osdp.osdp_split_linear_i8_workspace_bytes(T, I, O, N, 1)[1] == I * O
        assert osdp.osdp_split_linear_i8_workspace_bytes(T, I, 1 << 27, N, 8)[1] == I * (1 << 24)
    assert osdp.osdp_split_linear_i8_workspace_bytes(64, 112, (1 << 27) - 16, 7, 1)[1] == 0
    fits = (1 << 31) - 512
    assert osdp.osdp_split_linear_i8_workspace_bytes(1, 16, fits, 1, 1)[1] == 0
    for O in (fits + 8, (1 << 31) - 8):
        with pytest.raises(osdp.OsdpError) as e:
            osdp.osdp_split_linear_i8_workspace_bytes(1, 16, O, 1, 1)
        assert e.value.status == B.OSDP_ERR_UNSUPPORTED


def test_i8_quantize_refuses():
    def call(I=64, O=32, N=2, w=P, q=P, scale=P, ws=P, ws_bytes=1 << 30):
        shape = B.osdp_shape(0, I, O, N, 0)
        return osdp.lib.osdp_split_linear_i8_quantize(ctypes.byref(shape), (ctypes.c_void_p * 2)(P, w), (ctypes.c_void_p * 2)(P, q),
                                                      scale, ws, ws_bytes, None)
    assert call(w=None) == B.OSDP_ERR_INVALID_ARG and call(q=None) == B.OSDP_ERR_INVALID_ARG
    assert call(w=P + 2) == B.OSDP_ERR_UNSUPPORTED and call(q=P + 8) == B.OSDP_ERR_UNSUPPORTED
    assert call(scale=None) == B.OSDP_ERR_INVALID_ARG and call(scale=P + 4) == B.OSDP_ERR_UNSUPPORTED
    assert call(ws=None) == B.OSDP_ERR_INVALID_ARG and call(ws=P + 64) == B.OSDP_ERR_UNSUPPORTED
    assert call(ws_bytes=0) == B.OSDP_ERR_WORKSPACE and call(I=8) == B.OSDP_ERR_UNSUPPORTED and call(O=4) == B.OSDP_ERR_UNSUPPORTED
    assert osdp.osdp_split_linear_i8_quantize_workspace_bytes(4096, 16384, 8) >= 4 * 16384
    assert osdp.lib.osdp_split_linear_i8_quantize(None, None, None, None, None, 0, None) == B.OSDP_ERR_INVALID_ARG


def test_the_binding_refuses_before_it_calls():
    import torch
    with pytest.raises(osdp.OsdpError):
        osdp.AdamWTable()
    with pytest.raises(osdp.OsdpError):   # not on a GPU
        osdp.AdamWTable(grads=[torch.zeros(4)])
    with pytest.raises(osdp.OsdpError):
        osdp.AdamWTable(grads=[torch.zeros(4)], params=[])


def test_arrays_that_share_memory_are_found():
    import random
    rng = random.Random(3)
    found = 0
    for _ in range(2000):
        spans = lambda k: [(rng.randrange(60), rng.randrange(9)) for _ in range(k)]  # noqa: E731
        written, read = spans(rng.randrange(5)), spans(rng.randrange(4))
        meet = lambda x, y: x[1] and y[1] and x[0] < sum(y) and y[0] < sum(x)  # noqa: E731
        want = any(meet(x, y) for i, x in enumerate(written) for y in written[:i] + read)
        assert B._overlap(written, read) == bool(want), (written, read)
        found += bool(want)
    assert 400 < found < 1600


def test_the_binding_refuses_scalars_that_are_not_on_the_gpu():
    import torch

    class Table:
        tensors, count, grad_type, param_type, state_bits, lengths = None, 0, 0, 0, 8, [4]
    one = lambda kind: torch.ones(1, dtype=kind)  # noqa: E731
    for kw in (dict(grad_sumsq=one(torch.float64)), dict(step_device=one(torch.int64)), dict(lr_device=one(torch.float32))):
        with pytest.raises(osdp.OsdpError, match="on the GPU"):
            osdp.osdp_adamw_step(Table, lr=1e-3, **kw)
    with pytest.raises(osdp.OsdpError, match="on the GPU"):
        osdp.osdp_adamw_grad_sumsq(Table, one(torch.float64), one(torch.uint8))
    Table.count = 1
    out = [torch.zeros(4, dtype=torch.bfloat16)]
    with pytest.raises(osdp.OsdpError, match="on the GPU"):
        osdp.osdp_adamw_state_values(Table, out, out)


def test_the_binding_refuses_other_types_of_matrices():
    import torch
    z = lambda *n, d=torch.bfloat16: torch.zeros(*n, dtype=d)  # noqa: E731
    q, scale, ws = [z(16 * 16, d=torch.int8)], z(16, d=torch.float32), z(1 << 16, d=torch.uint8)
    for X, Y, s in ((z(2, 16, d=torch.float16), z(2, 16), scale), (z(2, 16), z(2, 16, d=torch.float16), scale), (z(2, 16), z(3, 16), scale),
                    (z(16, 2).t(), z(2, 16), scale), (z(2, 16), z(2, 16), z(8, d=torch.float32)), (z(2, 16), z(2, 16), z(16, d=torch.float64)),
                    (z(2, 16), z(2, 16), z(32, d=torch.float32)[::2])):
        with pytest.raises(osdp.OsdpError) as e:
            osdp.osdp_split_linear_i8_fwd(X, q, s, Y, 1, ws)
        assert e.value.status == B.OSDP_ERR_INVALID_ARG
    for w, qs, s in (([z(256)] * 2, q, scale), ([z(256)], q, z(15, d=torch.float32)), ([z(256)], q, z(16))):
        with pytest.raises(osdp.OsdpError) as e:
            osdp.osdp_split_linear_i8_quantize(16, 16, w, qs, s, ws)
        assert e.value.status == B.OSDP_ERR_INVALID_ARG


class OnGpu:
    """What the binding asks a tensor for, of one that would lie on a GPU."""
    def __init__(self, shape, dtype="bfloat16", device=0, contiguous=True, address=P):
        import torch
        self.shape = shape if isinstance(shape, tuple) else (shape,)
        self.dtype, self.device, self.contiguous, self.is_cuda = getattr(torch, dtype), device, contiguous, device >= 0
        self.nbytes, self.address = self.numel() * self.dtype.itemsize, address

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous

    def stride(self):
        return self.shape[-1], 1

    def data_ptr(self):
        return self.address if self.device >= 0 else 0


@pytest.fixture
def no_gpu_work(monkeypatch):
    """Calls that pass all checks, the binding's and the library's, end here with OSDP_ERR_HIP: there is no GPU to ask for."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a call that passes the checks would run")


@pytest.mark.parametrize("name", ["w_shards", "q_shards", "fwd"])
@pytest.mark.parametrize("bad", [dict(dtype="float32"), dict(dtype="float16"), dict(dtype="int16"), dict(n=-1), dict(device=-1), dict(device=1),
                                 dict(contiguous=False), dict(dtype="other")])
@pytest.mark.parametrize("place", [0, 2, 3])
def test_the_binding_refuses_other_shards(no_gpu_work, name, bad, place):
    I, O, N = 272, 24, 4
    L = I * O // N
    bad = dict(bad)
    if bad.get("dtype") == "other":   # the other matrix's shards
        bad["dtype"] = "int8" if name == "w_shards" else "bfloat16"
    w, q = [OnGpu(L) for _ in range(N)], [OnGpu(L, "int8") for _ in range(N)]
    scale, ws = OnGpu(O, "float32"), OnGpu(1 << 30, "uint8")

    def call():
        if name == "fwd":
            osdp.osdp_split_linear_i8_fwd(OnGpu((2, I)), q, scale, OnGpu((2, O), address=2 * P), 1, ws)
        else:
            osdp.osdp_split_linear_i8_quantize(I, O, w, q, scale, ws)
    with pytest.raises(osdp.OsdpError) as e:   # what is right gets as far as the GPU
        call()
    assert e.value.status in (B.OSDP_ERR_HIP, B.OSDP_ERR_UNSUPPORTED) and "aligned" not in str(e.value)
    shards = w if name == "w_shards" else q
    kind = dict(n=0, dtype="bfloat16" if name == "w_shards" else "int8")
    kind.update(bad)
    shards[place] = OnGpu(L + kind.pop("n"), **kind)
    with pytest.raises(osdp.OsdpError, match=r"_shards\[%d\]" % place) as e:
        call()
    assert e.value.status == B.OSDP_ERR_INVALID_ARG


def test_the_last_shard_may_hold_less_and_bytes_may_have_no_sign(no_gpu_work):
    """112 x 8 elements in 19 shards of 48, of which the last holds 32; 16 x 16 in 17 of 16, of which the last holds none."""
    for I, O, N, L in ((112, 8, 19, 48), (16, 16, 17, 16)):
        for kind in ("int8", "uint8"):
            for less in (0, 1):
                q = [OnGpu(L, kind) for _ in range(N - 1)] + [OnGpu(max(I * O - (N - 1) * L - less, 0), kind)]
                with pytest.raises(osdp.OsdpError) as e:
                    osdp.osdp_split_linear_i8_fwd(OnGpu((2, I)), q, OnGpu(O, "float32"), OnGpu((2, O), address=2 * P), 1, OnGpu(1 << 30, "uint8"))
                assert ("q_shards[18]" in str(e.value)) == bool(less and N == 19), e.value


def test_the_look_at_shards_leaves_to_python_what_it_cannot_answer():
    import torch
    look, kinds = B._checked_pointers, bytes((0, 8))
    assert look([], 64, kinds, 0) == b""
    for ts in ([torch.zeros(64, dtype=torch.int8)], (torch.zeros(64),), [OnGpu(64, "int8")], [None], [3, "x"],
               [torch.zeros(4).to_sparse()], [torch.zeros(64, dtype=torch.int8, device="meta")]):
        assert look(ts, 1, kinds, 0) is None
    for args in (([], 1, kinds), ([], 1, "x", 0), (3, 1, kinds, 0), ([], "1", kinds, 0), ([], 1, kinds, None), ([], 1 << 70, kinds, 0)):
        with pytest.raises((TypeError, OverflowError)):
            look(*args)


@pytest.mark.parametrize("place", ["X", "Y", "scale", "ws"])
@pytest.mark.parametrize("device", [-1, 1])
def test_the_binding_refuses_other_devices(no_gpu_work, place, device):
    I, O = 64, 32
    at = {name: device if name == place else 0 for name in ("X", "Y", "scale", "ws")}
    args = dict(X=OnGpu((2, I), device=at["X"]), Y=OnGpu((2, O), device=at["Y"]), scale=OnGpu(O, "float32", at["scale"]),
                ws=OnGpu(1 << 30, "uint8", at["ws"]))
    q, w = [OnGpu(I * O, "int8")], [OnGpu(I * O)]
    with pytest.raises(osdp.OsdpError, match="GPU") as e:
        osdp.osdp_split_linear_i8_fwd(args["X"], q, args["scale"], args["Y"], 1, args["ws"])
    assert e.value.status == B.OSDP_ERR_INVALID_ARG
    if place in ("scale", "ws"):
        with pytest.raises(osdp.OsdpError, match="GPU") as e:
            osdp.osdp_split_linear_i8_quantize(I, O, w, q, args["scale"], args["ws"])
        assert e.value.status == B.OSDP_ERR_INVALID_ARG


def test_new_gradients_may_not_share_memory_with_what_is_written():
    """set_grads refuses what the constructor does."""
    at = lambda name, i: P * (1 + ("param", "master", "m", "v", "exps", "grad").index(name)) + 4096 * i  # noqa: E731
    make = lambda name, n, kind: [OnGpu(n, kind, address=at(name, i)) for i in range(2)]  # noqa: E731
    table = osdp.AdamWTable(params=make("param", 256, "bfloat16"), grads=make("grad", 256, "bfloat16"), masters=make("master", 256, "float32"),
                            m=make("m", 256, "uint8"), v=make("v", 256, "uint8"), exps=make("exps", 4, "uint8"))
    bf16 = lambda address: OnGpu(256, address=address)  # noqa: E731
    before = [table.tensors[i].grad for i in range(2)]
    sizes = dict(param=512, master=1024, m=256, v=256, exps=4)
    for name, size in sizes.items():
        for i in range(2):
            for bad in (at(name, i), at(name, i) + size - 2, at(name, i) - 510):
                for place in range(2):
                    new = [bf16(1 << 30), bf16(1 << 30)]
                    new[place] = bf16(bad)
                    with pytest.raises(osdp.OsdpError, match="share memory"):
                        table.set_grads(new)
                    assert [table.tensors[i].grad for i in range(2)] == before
            table.set_grads([bf16(at(name, i) + size), bf16(at(name, i) - 512)])   # side by side
            before = [table.tensors[i].grad for i in range(2)]
    table.set_grads([bf16(1 << 30), bf16(1 << 30)])                                # read twice


def test_a_table_and_its_scalars_are_on_one_gpu(no_gpu_work):
    def lists(place=None, device=1):
        at = lambda i, n, kind, name: OnGpu(n, kind, device if (name, i) == place else 0, address=P * (1 + 2 * len(name) + i) + 4096 * ord(name[0]))  # noqa: E731
        pair = lambda name, n, kind: [at(i, n, kind, name) for i in range(2)]  # noqa: E731
        return dict(params=pair("params", 256, "bfloat16"), grads=pair("grads", 256, "bfloat16"), masters=pair("masters", 256, "float32"),
                    m=pair("m", 256, "uint8"), v=pair("v", 256, "uint8"), exps=pair("exps", 4, "uint8"))
    for name in lists():
        for i in range(2):
            with pytest.raises(osdp.OsdpError, match="GPU") as e:
                osdp.AdamWTable(**lists((name, i)))
            assert e.value.status == B.OSDP_ERR_INVALID_ARG
    table = osdp.AdamWTable(**lists())
    with pytest.raises(osdp.OsdpError, match="GPU"):
        table.set_grads(lists(("grads", 1))["grads"])
    away = lambda kind: OnGpu(1, kind, 1)  # noqa: E731
    for kw in (dict(grad_sumsq=away("float64")), dict(step_device=away("int64")), dict(lr_device=away("float32"))):
        with pytest.raises(osdp.OsdpError, match="on the GPU"):
            osdp.osdp_adamw_step(table, lr=1e-3, **kw)
    with pytest.raises(osdp.OsdpError, match="on the GPU"):
        osdp.osdp_adamw_grad_sumsq(table, away("float64"), OnGpu(1024, "uint8", 1))
    here, there = ([OnGpu(256, device=d, address=(30 + i) * P) for i in range(4)] for d in (0, 1))
    for m_out, v_out in ((here[:2], there[2:]), (there[:2], here[2:])):
        with pytest.raises(osdp.OsdpError, match="on the GPU"):
            osdp.osdp_adamw_state_values(table, m_out, v_out)


def test_the_sum_of_squares_refuses_a_workspace_that_is_not_on_the_gpu():
    class Table:
        tensors, count, grad_type = (B.osdp_adamw_tensor * 1)(), 0, 0
    for ws in (OnGpu(1024, "uint8", -1), OnGpu(1024, "uint8", 0, False)):
        with pytest.raises(osdp.OsdpError, match="workspace must be"):
            osdp.osdp_adamw_grad_sumsq(Table, OnGpu(1, "float64"), ws)


def test_rounding_by_one_multiplication_and_one_addition_is_exact():
    """trunc(fma(x, r, 1/2)), r = fp32(fp32(127 / amax) (1 + 2^-21)), against round(x * 127 / amax), halves upwards, in whole numbers: for every
    significand of a bf16 x and amax at every power of two between them that leaves something."""
    import numpy as np
    a, b = np.meshgrid(np.arange(128, 256, dtype=np.int64), np.arange(128, 256, dtype=np.int64), indexing="ij")
    r = (np.float32(127) / b.astype(np.float32)) * np.float32(1 + 2.0 ** -21)
    assert r.dtype == np.float32
    for j in range(12):
        ok = a <= b * 2 ** j            # x = a 2^-j is no larger than amax = b
        exact = (2 * 127 * a + b * 2 ** j) // (2 * b * 2 ** j)
        t = (a * 2.0 ** -j * r.astype(np.float64) + 0.5).astype(np.float32)  # (32 bits of product and a half: exact in 64, rounded once)
        assert (t.astype(np.int64) == exact)[ok].all(), j
        assert t[ok].max() < 128
