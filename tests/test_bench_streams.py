"""What bench.py times of AdamW and the 8-bit operator: on the step's own streams, after what was prepared on another one."""
from types import SimpleNamespace

import pytest

import bench


class Log:
    """Stands for torch and for the library: notes what is called, and on which stream."""
    def __init__(self):
        self.calls = []
        log = self

        class Event:
            def __init__(self, **kw):
                pass

            def record(self, stream=None):
                log.calls.append(("record", stream, None))

            def elapsed_time(self, other):
                return 1.0
        array = SimpleNamespace(numel=lambda: 64, float=lambda: array)
        make = lambda *a, **kw: (self.calls.append(("make", None, None)), array)[1]  # noqa: E731
        self.torch = SimpleNamespace(empty=make, zeros=make, float32="f", float64="d", uint8="u", int8="i",
                                     cuda=SimpleNamespace(Event=Event, synchronize=lambda: self.calls.append(("synchronize", None, None))))
        self.array = array

    def __getattr__(self, name):
        if not name.startswith("osdp_"):
            return {"OSDP_ADAMW_BLOCK": 128, "AdamWTable": lambda **kw: None}[name]
        if name.endswith("_bytes"):
            return lambda *a, **kw: (64, 0) if "quantize" not in name and "split" in name else 64
        return lambda *a, **kw: self.calls.append((name, kw.get("stream", kw.get("stream_compute")), kw.get("stream_copy")))


def stack(mixed):
    log = Log()
    st = bench.Stack.__new__(bench.Stack)
    st.torch, st.osdp, st.sc, st.sp, st.mixed, st.ws, st.plan = log.torch, log, "compute", "copy", mixed, None, None
    op = SimpleNamespace(I=8, O=8, k=2)
    st.w = SimpleNamespace(T=4, N=1, ops=[op], layers=1)
    st.ops = [dict(op=op, n=0, W=[log.array], dW=[log.array], X=0, Y=0, dX=0, dY=0, w_dp=0, dw_dp=0)]
    return st, log


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("which", ["adamw 32", "adamw 8", "int8"])
def test_work_is_timed_on_the_streams_of_a_step(which, mixed):
    st, log = stack(mixed)
    if which == "int8":
        bench.int8_forward(st, 3, 1)
    else:
        bench.training_step(st, int(which[6:]), 3, 1)
    names = [c[0] for c in log.calls]
    work = [c for c in log.calls if c[0].startswith("osdp_") or c[0] == "record"]
    assert work and all(stream == "compute" for _, stream, _ in work), work
    passes = [c for c in work if "split_linear_fwd" in c[0] or "split_linear_bwd" in c[0]]
    assert passes and all(copy == "copy" for _, _, copy in passes), "without its copy stream a pass is not what a step runs"
    assert all(("mixed" in c[0]) == mixed for c in passes)
    last = max(i for i, n in enumerate(names) if n == "make")
    first = min(i for i, n in enumerate(names) if n.startswith("osdp_"))
    assert "synchronize" in names[last:first], "what is filled on another stream has to be there first"
