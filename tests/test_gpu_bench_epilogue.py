"""What bench.py times of the step with biases, activations, residuals and heads: that it runs, and on what the workload holds."""
import pytest
import torch

import bench
import paper_2209_13258_amd as osdp
import workloads as wl

pytestmark = pytest.mark.gpu


def test_the_step_of_a_layer_with_epilogues_runs():
    w = wl.Workload(0, "layer", 300, 4, wl._layer(256, 512, (2, 1, 2, 2)), 1, ())
    st = bench.Stack(w, osdp.OSDP_STAGING_AUTO, torch, osdp)
    got = bench.epilogue_step(st, 3, 1)
    assert got["median_ms_per_step"] > 0 and got["tflops"] > 0 and got["products_alone_ms_per_step"] > 0
    torch.cuda.synchronize()
    assert all(torch.isfinite(t).all() for d in st.ops for t in [d["Y"], d["dX"], *d["dW"]])
