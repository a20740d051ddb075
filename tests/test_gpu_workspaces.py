"""Workspaces of the runners and torch's allocator: a runner dropped behind a run on another stream than its own gives its memory back
only when that run is over."""
import pytest

from paper_2002_12418_b200 import binding as B
from paper_2002_12418_b200 import workloads as W

pytestmark = pytest.mark.gpu


def linear(torch):
    x, w = torch.ones(1500, 640, device="cuda"), torch.ones(1300, 640, device="cuda")
    r = B.LinearRunner(1500, 1300, 640)
    assert r.info.workspace_bytes > 1 << 20
    return r, (lambda y: r.run(x, w, y=y)), (x, w), torch.empty(1500, 1300, device="cuda"), 640.0


def conv(torch):
    x, w = torch.ones(8, 64, 30, 30, device="cuda"), torch.ones(64, 64, 3, 3, device="cuda")
    r = B.ConvLayerRunner(8, 64, 64, 30, 30, 3, 1, 0, 1, B.make_opts(force_algo=B.ALGO_WINOGRAD, force_m=4, fused=1))
    assert r.info.workspace_bytes > 1 << 20
    r.prepare(w)
    return r, (lambda y: r.run(x, w, y=y)), (x, w), torch.empty(8, 64, 28, 28, device="cuda"), 576.0


def net(torch):
    layers = [W.ConvLayer("a", 8, 64, 64, 30, 30, 1, 1, 0, seed=1), W.ConvLayer("b", 8, 64, 64, 30, 30, 1, 1, 0, seed=2)]
    ws = [torch.full((64, 64, 1, 1), 1.0 / 64.0, device="cuda") for _ in layers]
    x = torch.ones(8, 64, 30, 30, device="cuda")
    r = B.NetRunner(8, 30, 30, layers)
    assert r.info.workspace_bytes > 1 << 20
    r.prepare(ws)
    r.bind(ws, [None, None])
    return r, (lambda y: r.run(x, y)), (x, ws), torch.empty(8, 64, 30, 30, device="cuda"), 1.0


@pytest.mark.parametrize("make", [linear, conv, net])
def test_memory_of_a_dropped_runner_waits_for_its_run(make):
    import torch
    r, run, inputs, y, want = make(torch)            # (the inputs stay: they are the caller's)
    size, at = r.workspace.numel(), r.workspace.data_ptr()
    side = torch.cuda.Stream()
    run(y)                                           # (kernels are loaded at their first launch, which waits for the device)
    torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)
    with torch.cuda.stream(side):
        torch.cuda._sleep(1000)
    y.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)             # some 0.5 s, in which the run below cannot begin
        run(y)
    del r, run
    taken = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255) for _ in range(2)]
    assert not side.query(), "the run was over too soon for this test to say anything"
    assert all(t.data_ptr() != at for t in taken)
    torch.cuda.synchronize()
    assert torch.allclose(y, torch.full_like(y, want), rtol=1e-3)


def test_a_runner_built_on_a_stream_leaves_its_memory_s_last_user_alone():
    import torch
    r = B.LinearRunner(4, 8, 16)
    size = r.workspace.numel()
    x, w = torch.ones(4, 16, device="cuda"), torch.ones(8, 16, device="cuda")
    r.run(x, w)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.empty(size, dtype=torch.uint8, device="cuda").fill_(77).clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        first = torch.empty(size, dtype=torch.uint8, device="cuda").fill_(77)
        at = first.data_ptr()
        torch.cuda._sleep(200_000_000)
        copy = first.clone()
        del first
        r2 = B.LinearRunner(4, 8, 16)                # takes the memory that `first` had, which the copy has not read yet
        assert r2.workspace.data_ptr() == at
        y = r2.run(x, w)
    torch.cuda.synchronize()
    assert (copy == 77).all() and (y == 16).all() and r2.device_status() == 0


def test_a_subclass_s_stream_is_recorded():
    import torch
    side = torch.cuda.Stream()

    class OnSide(B.LinearRunner):
        def stream(self):
            return side.cuda_stream

    x, w, y = torch.ones(1500, 640, device="cuda"), torch.ones(1300, 640, device="cuda"), torch.empty(1500, 1300, device="cuda")
    r = OnSide(1500, 1300, 640)
    size, at = r.workspace.numel(), r.workspace.data_ptr()
    torch.cuda.synchronize()
    r.run(x, w, y=y)
    torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    y.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)
    r.run(x, w, y=y)
    del r
    taken = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255) for _ in range(2)]
    assert not side.query() and all(t.data_ptr() != at for t in taken)
    torch.cuda.synchronize()
    assert (y == 640).all()
