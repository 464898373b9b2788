"""Calibration on a given stream takes its workspace from that stream's blocks."""
import numpy as np
import pytest

from paper_2609_38169_gb300 import api as A, workloads as W

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_the_workspace_belongs_to_the_stream_of_the_call(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    wl = W.WORKLOADS["tiny"].replace(layers=1, hk=2, hv=2)
    cfg = A.Config.from_workload(wl)
    mp = W.model_params_torch(W.model_params(wl), "cuda")
    steps = [W.torch_step_inputs(wl, mp, t, 0, "cuda", W.STREAM_CALIB, batch=2) for t in range(6)]
    trace = [torch.stack([s[i] for s in steps])[None].contiguous() for i in range(5)]
    side, seen, empty = torch.cuda.Stream(), [], torch.empty
    torch.cuda.synchronize()

    def watched(*a, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **kw)

    monkeypatch.setattr(torch, "empty", watched)
    got = [A.stepq_calibrate_from_trace(cfg, *trace, every=3, stream=s) for s in (None, side)]
    assert seen == [torch.cuda.current_stream().cuda_stream, side.cuda_stream]
    np.testing.assert_allclose(got[0].omega, got[1].omega, rtol=2e-7)     # fp64 sums in any order, rounded
    np.testing.assert_allclose(got[0].dist, got[1].dist, rtol=1e-12)
