"""Calls that are given no workspace: under a stream capture, and where torch has no memory left."""
import ctypes
import sys

import numpy as np
import pytest

from paper_2303_10384_amd import workloads as W
from test_gpu_parity import pkg, to_dev, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def announce(request):
    sys.__stderr__.write("\n[gpu-test] %s\n" % request.node.nodeid)
    sys.__stderr__.flush()
    yield


def inputs(torch):  # noqa: F811
    logits, tl, ul, labels = W.small_case(6, 20, 9, 48, seed=8, sigma=2.0)
    return [to_dev(torch, a) for a in (logits, labels, tl, ul)]


class Capture:
    """A capture that torch did not begin: HIP's own calls on a torch stream."""

    def __init__(self, torch):  # noqa: F811
        self.hip = ctypes.CDLL("libamdhip64.so")
        self.stream = torch.cuda.Stream()
        self.raw = ctypes.c_void_p(self.stream.cuda_stream)

    def check(self, code):
        assert code == 0, code

    def record(self, torch, fn):  # noqa: F811
        graph, self.exec = ctypes.c_void_p(), ctypes.c_void_p()
        with torch.cuda.stream(self.stream):
            self.check(self.hip.hipStreamBeginCapture(self.raw, 2))  # relaxed
            fn()
            self.check(self.hip.hipStreamEndCapture(self.raw, ctypes.byref(graph)))
        self.check(self.hip.hipGraphInstantiate(ctypes.byref(self.exec), graph, None, None, ctypes.c_size_t(0)))

    def replay(self):
        self.check(self.hip.hipGraphLaunch(self.exec, self.raw))


def test_capture_that_torch_did_not_begin(torch, pkg):  # noqa: F811
    lg, labels, tl, ul = inputs(torch)
    grad, loss = torch.empty_like(lg), torch.empty(6, dtype=torch.float32, device="cuda")

    def call():
        pkg.rnnt_loss(lg, labels, tl, ul, variant="wrnnt", grad_out=grad, loss_out=loss)

    call()
    torch.cuda.synchronize()
    loss_ref, grad_ref = loss.clone(), grad.clone()
    c = Capture(torch)
    c.record(torch, call)
    n = pkg.loss_workspace_bytes(6, 20, 9, 48)
    # blocks of the workspace's size, allocated after the capture on its stream: a replay must not write them
    with torch.cuda.stream(c.stream):
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(3):
        grad.fill_(float("nan"))
        loss.fill_(float("nan"))
        torch.cuda.synchronize()
        c.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, loss_ref) and torch.equal(grad, grad_ref)
        assert all(bool((o == 7).all()) for o in others)
        call()  # eager work between the replays
        torch.cuda.synchronize()


def test_torch_graph_without_a_workspace(torch, pkg):  # noqa: F811
    lg, labels, tl, ul = inputs(torch)
    loss_ref, grad_ref = pkg.rnnt_loss(lg, labels, tl, ul)
    grad, loss = torch.empty_like(lg), torch.empty_like(loss_ref)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pkg.rnnt_loss(lg, labels, tl, ul, grad_out=grad, loss_out=loss)
    for _ in range(3):
        grad.fill_(float("nan"))
        loss.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, loss_ref) and torch.equal(grad, grad_ref)
        pkg.rnnt_loss(lg, labels, tl, ul, grad_out=grad, loss_out=loss)
        torch.cuda.synchronize()


def test_no_memory_left_in_torch(torch, pkg, monkeypatch):  # noqa: F811
    """torch's allocator refusing the workspace is not an error of the call: the library's own checks come
    first, and it takes a workspace of its own."""
    lg, labels, tl, ul = inputs(torch)
    loss_ref, grad_ref = pkg.rnnt_loss(lg, labels, tl, ul)
    grad, loss = torch.empty_like(lg), torch.empty_like(loss_ref)
    empty = torch.empty

    def no_bytes(*args, **kw):
        if kw.get("dtype") is torch.uint8:
            raise torch.OutOfMemoryError("no memory left")
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", no_bytes)
    pkg.rnnt_loss(lg, labels, tl, ul, grad_out=grad, loss_out=loss)
    assert torch.equal(loss, loss_ref) and torch.equal(grad, grad_ref)
    xr = lg.clone().requires_grad_(True)
    pkg.RNNTLoss(reduction="sum")(xr, labels, tl, ul).backward()
    assert np.array_equal(xr.grad.cpu().numpy(), grad_ref.cpu().numpy())
    with pytest.raises(pkg.RNNTError, match="blank"):
        pkg.rnnt_loss(lg, labels, tl, ul, blank=99, grad_out=grad, loss_out=loss)


def test_captured_call_without_a_workspace_is_refused(torch, pkg):  # noqa: F811
    """The C calls: none is allocated inside a capture, which goes on; eager calls take their own."""
    from paper_2303_10384_amd import binding
    lg, labels, tl, ul = inputs(torch)
    loss_ref, grad_ref = pkg.rnnt_loss(lg, labels, tl, ul)
    lib, shape = binding.load_library(), binding.shape_of(lg)
    loss, grad = torch.zeros_like(loss_ref), torch.zeros_like(lg)
    ptr = lambda t: t.data_ptr()  # noqa: E731

    def call():
        return lib.rnnt_loss(ptr(lg), shape, ptr(labels), ptr(tl), ptr(ul), 0, 0, ptr(loss), ptr(grad), None, 0,
                             torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        status = call()
        loss.fill_(3.0)
    assert status == 6
    g.replay()
    torch.cuda.synchronize()
    assert bool((loss == 3).all()) and bool((grad == 0).all())
    assert call() == 0
    torch.cuda.synchronize()
    assert torch.equal(loss, loss_ref) and torch.equal(grad, grad_ref)


def test_captured_autograd_loss(torch, pkg):  # noqa: F811
    """Loss and gradient through autograd in a graph, with memory of torch's alone; the upstream gradient and the
    logits change between the replays."""
    lg, labels, tl, ul = inputs(torch)
    up = torch.ones(6, device="cuda")
    lg.requires_grad_(True)

    def step():
        loss = pkg.rnnt_loss_autograd(lg, labels, tl, ul, reduction="none")
        return loss.detach(), torch.autograd.grad(loss, lg, up)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        up.fill_(1.0 + i)
        with torch.no_grad():
            lg.mul_(1.125)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_refused_allocation_is_not_the_next_calls_error(torch, pkg):  # noqa: F811
    """A workspace of 8.8 TB, which the runtime refuses, is this call's status 8; the next call is not told of it."""
    net = pkg.network
    lib = net._library()
    x = torch.ones(1 << 12, dtype=torch.bfloat16, device="cuda")
    lens = torch.ones(16, dtype=torch.int32, device="cuda")
    huge = net.JointShape(16, 8191, (1 << 18) - 1, 1024, 1)
    assert lib.rnnt_joint_hidden_grad_workspace_bytes(huge) > 1 << 42
    p, q, stream = x.data_ptr(), lens.data_ptr(), torch.cuda.current_stream().cuda_stream
    torch.cuda.synchronize()
    assert lib.rnnt_joint_hidden_grad(p, p, huge, q, q, 0, 0.0, None, p, p, p, None, 0, stream) == 8
    y = pkg.dropout(x, 0.0, torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert torch.equal(x, y)


def test_every_call_captured_without_a_workspace(torch, pkg):  # noqa: F811
    """Alignment, lattice scores, the loss over arc lists and the loss, with results of their own, in one graph: each
    call's workspace lives with a result of it."""
    lg, labels, tl, ul = inputs(torch)
    lab, t, u = (a.cpu().numpy() for a in (labels, tl, ul))
    lattices = [pkg.topologies.grid_lattice(int(t[b]), int(u[b]), lab[b, :u[b]], variant="rnnt") for b in range(6)]
    plan = pkg.arc_plan(lattices, 20, 9, 48, blank=0, device="cuda")
    _, lp_blank, lp_label = pkg.log_softmax_gather(lg, labels, tl, ul)

    def call():
        scores = pkg.lattice_scores(lp_blank, lp_label, tl, ul)
        return (pkg.rnnt_loss(lg, labels, tl, ul) + pkg.viterbi_align(lg, labels, tl, ul) + pkg.arc_loss(lg, tl, ul, plan)
                + pkg.rnnt_loss(lg, labels, tl, ul, variant="wrnnt", need_grad=False)[:1]
                + tuple(scores[k] for k in sorted(scores)))

    want = [x.clone() for x in call()]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    for _ in range(3):
        for x in out:
            x.fill_(-7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(torch.nan_to_num(a.double(), 3e300), torch.nan_to_num(b.double(), 3e300))
        again = call()  # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(torch.nan_to_num(a.double(), 3e300), torch.nan_to_num(b.double(), 3e300))
                   for a, b in zip(again, want))
