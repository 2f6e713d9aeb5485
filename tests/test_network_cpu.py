"""The network operators without a GPU: the C-ABI's exports and refusals (every call below is
turned down before any HIP call), workspace sizes, and the binding's checks."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "rnnt_network_mi355x.h")).read()
FAKE = 1 << 20  # aligned, never dereferenced
vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def net():
    from paper_2303_10384_amd import binding, network
    if not os.path.exists(binding.LIB_PATH):
        from paper_2303_10384_amd import build
        build.build(verbose=False)
    return network


def test_header_and_exports(net):
    src = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
    names = sorted(set(re.findall(r"\b(rnnt_[a-z_0-9]+)\s*\(", src)))
    assert names == sorted(net.EXPORTED)
    lib = net._library()
    for name in names:
        assert hasattr(lib, name), name
    assert int(re.search(r"#define RNNT_RECURRENCE_STATE_STEPS (\d+)", HEADER).group(1)) == net.STATE_STEPS


def call(fn, defaults, over):
    """fn on `defaults` (name -> value, in order) with some replaced."""
    args = dict(defaults)
    for k, v in over.items():
        assert k in args, k
        args[k] = v
    return fn(*args.values())


def test_embedding_refusals(net):
    lib, S = net._library(), net.EmbeddingShape
    ok = S(2, 3, 7, 5, 0, 0)
    fwd = {"labels": FAKE, "lens": FAKE, "shape": ok, "weight": FAKE, "scale": 1.0, "out": FAKE, "stream": None}
    for shape, want in ((S(0, 3, 7, 5, 0, 0), 2), (S(2, -1, 7, 5, 0, 0), 2), (S(2, 3, 0, 5, -1, 0), 2),
                        (S(2, 3, 7, 0, 0, 0), 2), (S(2, 3, 7, 5, 7, 0), 2), (S(2, 3, 7, 5, -2, 0), 2),
                        (S(2, 3, 7, 5, 0, 3), 4), (S(1 << 16, 1 << 15, 7, 5, -1, 0), 9)):
        assert call(lib.rnnt_label_embedding, fwd, {"shape": shape}) == want
        assert lib.rnnt_label_embedding_grad_workspace_bytes(shape) == 0
    for over, want in (({"labels": None}, 1), ({"weight": None}, 1), ({"out": None}, 1), ({"weight": FAKE + 2}, 7),
                       ({"out": FAKE + 1}, 7)):
        assert call(lib.rnnt_label_embedding, fwd, over) == want
    assert call(lib.rnnt_label_embedding, fwd, {"shape": S(2, 0, 7, 5, -1, 0), "labels": None, "out": None}) == 0
    need = lib.rnnt_label_embedding_grad_workspace_bytes(ok)
    assert need > 0 and need % 256 == 0
    bwd = {"labels": FAKE, "lens": FAKE, "shape": ok, "dout": FAKE, "scale": 1.0, "dweight": FAKE, "ws": FAKE,
           "bytes": need - 1, "stream": None}
    for over, want in (({}, 6), ({"dout": None}, 1), ({"dweight": None}, 1), ({"dout": FAKE + 2}, 7),
                       ({"ws": FAKE + 16, "bytes": need}, 7), ({"labels": None}, 1)):
        assert call(lib.rnnt_label_embedding_grad, bwd, over) == want


def test_embedding_sizes_past_a_launch(net):
    """Refused before the call's first launch (9), not by it (8)."""
    lib, S = net._library(), net.EmbeddingShape
    fwd = {"labels": FAKE, "lens": FAKE, "shape": S(2, 3, 1, 2 ** 31 - 1, 0, 0), "weight": FAKE, "scale": 1.0, "out": FAKE,
           "stream": None}
    assert call(lib.rnnt_label_embedding, fwd, {}) == 9
    bwd = {"labels": FAKE, "lens": FAKE, "shape": None, "dout": FAKE, "scale": 1.0, "dweight": FAKE, "ws": FAKE,
           "bytes": 1 << 62, "stream": None}
    for shape in (S(2, 3, 2 ** 31 - 1, 1, 0, 0), S(2, 3, 1 << 27, 4, -1, 1), S(1 << 14, 1 << 15, 2, 1024, -1, 0),
                  S(2, 3, 1, 2 ** 31 - 1, 0, 2)):
        assert call(lib.rnnt_label_embedding_grad, bwd, {"shape": shape}) == 9


def test_recurrence_refusals(net):
    lib, S = net._library(), net.RecurrenceShape
    assert lib.rnnt_recurrence_workspace_bytes(S(2, 40, 5, 0, 200, 5, 200, 5)) == 0  # one block to a sequence
    ok = S(2, 4000, 5, 0, 20000, 5, 20000, 5)
    need = lib.rnnt_recurrence_workspace_bytes(ok)
    assert need > 0 and need % 256 == 0
    assert lib.rnnt_recurrence_states_bytes(ok) == 2 * -(-4000 // net.STATE_STEPS) * 5 * 4
    fwd = {"x": FAKE, "z": FAKE, "shape": ok, "lens": FAKE, "h0": FAKE, "h": FAKE, "last": FAKE, "states": FAKE,
           "ws": FAKE, "bytes": need - 1, "stream": None}
    bwd = {"x": FAKE, "z": FAKE, "shape": ok, "lens": FAKE, "states": FAKE, "dh": FAKE, "dlast": FAKE, "dx": FAKE,
           "dz": FAKE, "dh0": FAKE, "ws": FAKE, "bytes": need - 1, "stream": None}
    for shape, want in ((S(0, 4, 5, 0, 20, 5, 20, 5), 2), (S(2, -1, 5, 0, 20, 5, 20, 5), 2),
                        (S(2, 4, 0, 0, 20, 5, 20, 5), 2), (S(2, 4, 5, 0, -20, 5, 20, 5), 2),
                        (S(2, 4, 5, 0, 20, 5, 20, -5), 2), (S(2, 4, 5, 9, 20, 5, 20, 5), 4)):
        assert call(lib.rnnt_recurrence, fwd, {"shape": shape}) == want
        assert call(lib.rnnt_recurrence_grad, bwd, {"shape": shape}) == want
        assert lib.rnnt_recurrence_workspace_bytes(shape) == lib.rnnt_recurrence_states_bytes(shape) == 0
    for over, want in (({}, 6), ({"x": None}, 1), ({"z": None}, 1), ({"h": None}, 1), ({"last": None}, 1),
                       ({"x": FAKE + 2}, 7), ({"h0": FAKE + 2}, 7), ({"last": FAKE + 1}, 7), ({"states": FAKE + 8}, 7),
                       ({"ws": FAKE + 16, "bytes": need}, 7)):
        assert call(lib.rnnt_recurrence, fwd, over) == want
    for over, want in (({}, 6), ({"x": None}, 1), ({"states": None}, 1), ({"dx": None}, 1), ({"dz": None}, 1),
                       ({"dh": FAKE + 2}, 7), ({"dlast": FAKE + 2}, 7), ({"dh0": FAKE + 2}, 7),
                       ({"dh": None, "dlast": None, "dh0": None}, 6)):
        assert call(lib.rnnt_recurrence_grad, bwd, over) == want


def test_dropout_refusals(net):
    lib = net._library()
    fwd = {"x": FAKE, "n": 0, "dtype": 0, "p": 0.5, "rng": FAKE, "rng_out": None, "y": FAKE, "stream": None}
    for over, want in (({"n": -1}, 2), ({"dtype": 3}, 4), ({"p": 1.0}, 5), ({"p": -0.1}, 5), ({"p": float("nan")}, 5),
                       ({"rng": None}, 1), ({"n": 4, "x": None}, 1), ({"n": 4, "y": None}, 1), ({"x": FAKE + 2}, 7),
                       ({"rng": FAKE + 4}, 7), ({"rng_out": FAKE + 4}, 7), ({"n": 1 << 62}, 9)):
        assert call(lib.rnnt_dropout, fwd, over) == want


def test_joint_refusals(net):
    lib, S = net._library(), net.JointShape
    ok = S(2, 4, 3, 5, 0)
    fwd = {"enc": FAKE, "pred": FAKE, "shape": ok, "tl": FAKE, "ul": FAKE, "act": 0, "p": 0.5, "rng": FAKE,
           "rng_out": None, "h": FAKE, "stream": None}
    need = lib.rnnt_joint_hidden_grad_workspace_bytes(ok)
    assert need > 0 and need % 256 == 0
    bwd = {"enc": FAKE, "pred": FAKE, "shape": ok, "tl": FAKE, "ul": FAKE, "act": 0, "p": 0.5, "rng": FAKE, "dh": FAKE,
           "denc": FAKE, "dpred": FAKE, "ws": FAKE, "bytes": need - 1, "stream": None}
    for shape, want in ((S(0, 4, 3, 5, 0), 2), (S(2, 0, 3, 5, 0), 2), (S(2, 4, -1, 5, 0), 2), (S(2, 4, 3, 0, 0), 2),
                        (S(2, 1 << 20, 1 << 20, 5, 0), 2), (S(2, 4, 3, 5, 3), 4)):
        assert call(lib.rnnt_joint_hidden, fwd, {"shape": shape}) == want
        assert call(lib.rnnt_joint_hidden_grad, bwd, {"shape": shape}) == want
        assert lib.rnnt_joint_hidden_grad_workspace_bytes(shape) == 0
    both = [({"enc": None}, 1), ({"pred": None}, 1), ({"tl": None}, 1), ({"ul": None}, 1), ({"act": 2}, 5),
            ({"p": 1.0}, 5), ({"p": -1.0}, 5), ({"p": float("nan")}, 5), ({"rng": None}, 1), ({"enc": FAKE + 2}, 7),
            ({"rng": FAKE + 4}, 7)]
    for over, want in both + [({"h": None}, 1), ({"h": FAKE + 1}, 7), ({"rng_out": FAKE + 4}, 7)]:
        assert call(lib.rnnt_joint_hidden, fwd, over) == want
    for over, want in both + [({}, 6), ({"dh": None}, 1), ({"denc": None}, 1), ({"dpred": None}, 1),
                              ({"dpred": FAKE + 2}, 7), ({"ws": FAKE + 16, "bytes": need}, 7)]:
        assert call(lib.rnnt_joint_hidden_grad, bwd, over) == want


def test_joint_sizes_past_a_launch(net):
    """Narrow rows (a thread to a channel) of more threads than a launch holds: refused, with nothing launched."""
    lib, S = net._library(), net.JointShape
    bwd = {"enc": FAKE, "pred": FAKE, "shape": None, "tl": FAKE, "ul": FAKE, "act": 0, "p": 0.5, "rng": FAKE, "dh": FAKE,
           "denc": FAKE, "dpred": FAKE, "ws": FAKE, "bytes": 1 << 62, "stream": None}
    for shape in (S(15, 1, (1 << 26) - 1, 7, 0), S(15, 1, (1 << 26) - 1, 7, 1), S(1 << 24, 16, 0, 3, 0)):
        assert call(lib.rnnt_joint_hidden_grad, bwd, {"shape": shape}) == 9


def test_binding_refuses_cpu_tensors_and_bad_arguments(net):
    import paper_2303_10384_amd as rnnt
    x, lens = torch.zeros(2, 3, 4), torch.ones(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        rnnt.label_embedding(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(5, 4))
    with pytest.raises(ValueError, match="GPU"):
        rnnt.gated_recurrence(x, x)
    with pytest.raises(ValueError, match="GPU"):
        rnnt.dropout(x, 0.5, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="GPU"):
        rnnt.joint_hidden(x, x, lens, lens)
    with pytest.raises(TypeError, match="tensor"):
        rnnt.dropout([1.0], 0.5, None)


def test_plain_forms_against_their_float64_results():
    """perf/operators.py on the CPU: its plain forms at half-step tolerances of their types."""
    import random
    from perf import operators as O
    rng = random.Random(11)
    cap = {"B": 3, "N": 20, "L": 40, "T": 7, "U": 5, "D": 40, "H": 40, "V": 50}
    for _ in range(16):
        case = {k: min(v, cap[k]) if k in cap else v for k, v in O.draw(rng).items()}
        got, want = O.run(O.prepare(case, 3)), O.exact(case, 3)
        got, want = (v if isinstance(v, tuple) else (v,) for v in (got, want))
        assert len(got) == len(want)
        for g, w in zip(got, want):
            step = torch.finfo(g.dtype).eps / 2
            # each element's own rounding, and float32 arithmetic on values of the tensor's size
            assert g.shape == w.shape
            assert bool(((g.double() - w).abs() <= step * w.abs() + 2.0 ** -18 * w.abs().max() + 1e-30).all()), case


# ---------------------------------------------------------------- the binding's calls, the library's stubbed

@pytest.fixture
def calls(net, monkeypatch):
    """The entry points on CPU tensors: every library call is recorded as (name, arguments) and does nothing."""
    made = []
    monkeypatch.setattr(net, "_check", lambda *args, **kw: None)
    monkeypatch.setattr(net, "_call", lambda fn, device, *args: made.append((fn.__name__, args)))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return made


def test_recurrence_gradient_of_tensors_saved_elsewhere(net, calls):
    """Hooks on saved tensors give backward copies of x and z laid out anew: the gradient's call names the strides
    of the copies, whose memory ends long before the strides of the views that the forward pass read would."""
    import paper_2303_10384_amd as rnnt
    both = torch.randn(2, 30, 12, requires_grad=True)
    lens = torch.tensor([30, 7], dtype=torch.int32)
    for copy in (lambda t: t.clone(memory_format=torch.contiguous_format),
                 lambda t: t if t.dim() != 3 else t.clone().transpose(1, 2).contiguous().transpose(1, 2)):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, copy):
            h, _ = rnnt.gated_recurrence(both[:, :, :6], both[:, :, 6:], None, lens)
            torch.autograd.grad(h, both, torch.ones_like(h))
        (_, fwd), (name, bwd) = calls[-2:]
        assert name == "rnnt_recurrence_grad"
        strides = lambda s: (s.x_stride_b, s.x_stride_t, s.z_stride_b, s.z_stride_t)  # noqa: E731
        assert strides(fwd[2]) == (360, 12, 360, 12) and strides(bwd[2]) == (180, 6, 180, 6)


def test_sizes_past_32_bits_are_refused(net, calls):
    """The descriptors hold 32-bit sizes: a larger one is an error, not its low half."""
    import paper_2303_10384_amd as rnnt
    wide = (1 << 32) + 8
    meta = lambda *s, **kw: torch.empty(s, device="meta", **kw)  # noqa: E731
    i32 = {"dtype": torch.int32}
    for call in (lambda: rnnt.label_embedding(meta(1, wide, **i32), meta(7, 4)),
                 lambda: rnnt.label_embedding(meta(1, 3, **i32), meta(wide, 4)),
                 lambda: rnnt.label_embedding(meta(1, 3, **i32), meta(7, wide, requires_grad=True)),
                 lambda: rnnt.gated_recurrence(meta(1, wide, 4), meta(1, wide, 4)),
                 lambda: rnnt.gated_recurrence(meta(wide, 1, 4), meta(wide, 1, 4)),
                 lambda: rnnt.joint_hidden(meta(1, wide, 4), meta(1, 1, 4), meta(1, **i32), meta(1, **i32)),
                 lambda: rnnt.joint_hidden(meta(1, 1, 4), meta(1, (1 << 31) + 1, 4), meta(1, **i32), meta(1, **i32))):
        with pytest.raises(rnnt.RNNTError, match="UNSUPPORTED"):
            call()
    assert not calls


def test_captured_losses_bring_their_workspace(net, monkeypatch):
    """Under a capture every loss call names a workspace (the library would have to refuse it without), which lives
    as long as a result does: behind the rows that backward needs, behind the losses, or with the caller's tensor."""
    import paper_2303_10384_amd as rnnt
    from paper_2303_10384_amd import binding
    real, made = binding.load_library(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes") or name == "rnnt_status_string":
                return getattr(real, name)
            return lambda *args: made.append((name, args)) or 0

    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "_check_gpu", lambda *args: None)
    monkeypatch.setattr(binding, "_stream_handle", lambda device: 0)
    monkeypatch.setattr(binding, "_capturing", lambda device: True)
    logits = torch.randn(2, 5, 4, 6, requires_grad=True)
    labels, tl, ul = torch.ones(2, 3, dtype=torch.int32), torch.full((2,), 5, dtype=torch.int32), torch.full((2,), 3, dtype=torch.int32)

    def inside(ptr, size, t):
        at = t.untyped_storage().data_ptr()
        return size > 0 and ptr % 256 == at % 256 and at + t.numel() * t.element_size() <= ptr and \
            ptr + size <= at + t.untyped_storage().nbytes()
    loss = rnnt.rnnt_loss_autograd(logits, labels, tl, ul)
    torch.autograd.grad(loss, logits, retain_graph=True)
    (name, fwd), (_, bwd) = made
    assert name == "rnnt_step_forward"
    rows = loss.grad_fn.saved_tensors[1]
    assert fwd[8] == bwd[3] == rows.data_ptr() and inside(fwd[9], fwd[10], rows)
    x = logits.detach()
    loss, _ = rnnt.rnnt_loss(x, labels, tl, ul)
    assert inside(made[-1][1][9], made[-1][1][10], loss)
    mine = torch.empty(2)
    rnnt.rnnt_loss(x, labels, tl, ul, loss_out=mine, grad_out=torch.empty_like(x))
    rnnt.rnnt_loss(x, labels, tl, ul, loss_out=mine, need_grad=False)
    assert [made[i][1][9] for i in (-2, -1)] == [w.data_ptr() for w in mine._captured_workspaces]
    score, _, _ = rnnt.viterbi_align(x, labels, tl, ul)
    assert made[-1][1][10] == score._captured_workspaces[0].data_ptr()
    given = torch.empty(1 << 20, dtype=torch.uint8)
    rnnt.rnnt_loss(x, labels, tl, ul, workspace=given)
    assert made[-1][1][9] == given.data_ptr()


def test_forward_mode_is_refused(net, calls):
    """A tensor that carries a tangent is an error, with and without requires_grad, not a result without one."""
    import torch.autograd.forward_ad as fw
    import paper_2303_10384_amd as rnnt
    x, w = torch.randn(2, 3, 4), torch.randn(5, 4)
    labels, lens, rng = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32), torch.tensor([1, 2])
    h0 = torch.randn(2, 4)
    with fw.dual_level():
        dual = lambda t, grad: fw.make_dual(t.clone().requires_grad_(grad), torch.ones_like(t))  # noqa: E731
        for grad in (False, True):
            for call in (lambda: rnnt.label_embedding(labels, dual(w, grad)), lambda: rnnt.gated_recurrence(dual(x, grad), x),
                         lambda: rnnt.gated_recurrence(x, dual(x, grad)), lambda: rnnt.gated_recurrence(x, x, dual(h0, grad)),
                         lambda: rnnt.dropout(dual(x, grad), 0.5, rng), lambda: rnnt.joint_hidden(dual(x, grad), x, lens, lens),
                         lambda: rnnt.joint_hidden(x, dual(x, grad), lens, lens)):
                with pytest.raises(NotImplementedError):
                    call()
                with pytest.raises(NotImplementedError), torch.no_grad():
                    call()
        n = len(calls)
        assert not rnnt.dropout(x, 0.5, rng).requires_grad and len(calls) == n + 1  # no tangent: as ever


def test_gradients_past_a_launch_are_refused_before_the_forward_call(net, calls):
    import paper_2303_10384_amd as rnnt
    meta = lambda *s, **kw: torch.empty(s, device="meta", **kw)  # noqa: E731
    i32, bf16 = {"dtype": torch.int32}, {"dtype": torch.bfloat16}
    lens = meta(64, **i32)
    for grad in (False, True):
        forward = ((lambda: rnnt.joint_hidden(meta(64, 25000, 640, **bf16, requires_grad=grad), meta(64, 1, 640, **bf16), lens, lens)),
                   (lambda: rnnt.joint_hidden(meta(1, 1, 8), meta(1, 1 << 26, 8, requires_grad=grad), meta(1, **i32), meta(1, **i32))),
                   (lambda: rnnt.joint_hidden(meta(1024, 16384, 16384, **bf16, requires_grad=grad), meta(1024, 1, 16384, **bf16),
                                              meta(1024, **i32), meta(1024, **i32))),
                   (lambda: rnnt.label_embedding(meta(2, 3, **i32), meta(1 << 27, 4, requires_grad=grad))))
        for i, make in enumerate(forward):
            n = len(calls)
            if grad and i != 0:
                with pytest.raises(rnnt.RNNTError, match="UNSUPPORTED"):
                    make()
                assert len(calls) == n
            else:
                make()
                assert len(calls) == n + 1
    lib = net._library()
    assert lib.rnnt_joint_hidden_grad_workspace_bytes(net.JointShape(1024, 16384, 0, 16384, 1)) == 0
    bwd = {"enc": FAKE, "pred": FAKE, "shape": net.JointShape(1024, 16384, 0, 16384, 1), "tl": FAKE, "ul": FAKE, "act": 0,
           "p": 0.5, "rng": FAKE, "dh": FAKE, "denc": FAKE, "dpred": FAKE, "ws": None, "bytes": 0, "stream": None}
    assert call(lib.rnnt_joint_hidden_grad, bwd, {}) == 9  # and no workspace is taken for it


def test_recurrence_states_in_place_are_refused(net):
    """Blocks that write the state would meet blocks that still read it."""
    lib = net._library()
    shape = net.RecurrenceShape(2, 8, 129, 1, 1032, 129, 1032, 129)  # needs no workspace
    size = 2 * 129 * 4
    for off in (0, 4, -4, size - 4, 4 - size):
        assert lib.rnnt_recurrence(FAKE, FAKE, shape, FAKE, FAKE, FAKE, FAKE + off, None, None, 0, None) == 9
        assert lib.rnnt_recurrence_grad(FAKE, FAKE, shape, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE + off, None, 0, None) == 9


def test_an_unknown_type_is_named(net, calls):
    import paper_2303_10384_amd as rnnt
    x, lens = torch.zeros(2, 3, 4, dtype=torch.float64), torch.ones(2, dtype=torch.int32)
    for name, call_it in (("weight", lambda: rnnt.label_embedding(torch.zeros(2, 3, dtype=torch.int32), x[0])),
                          ("x", lambda: rnnt.gated_recurrence(x, x)),
                          ("x", lambda: rnnt.dropout(x, 0.5, torch.zeros(2, dtype=torch.int64))),
                          ("enc", lambda: rnnt.joint_hidden(x, x, lens, lens))):
        with pytest.raises(TypeError, match="^%s must be float32, bfloat16 or float16, got torch.float64" % name):
            call_it()
