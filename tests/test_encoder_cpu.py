"""The encoder's operators without a GPU: the C-ABI's exports and refusals (every call below is
turned down before any HIP call), workspace sizes, the arithmetic of pages, and the binding's
checks."""
import ctypes
import itertools
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "rnnt_encoder_mi355x.h")).read()
FAKE = 1 << 20  # aligned, never dereferenced


@pytest.fixture(scope="module")
def enc():
    from paper_2303_10384_amd import binding, encoder
    if not os.path.exists(binding.LIB_PATH):
        from paper_2303_10384_amd import build
        build.build(verbose=False)
    return encoder


def test_header_and_exports(enc):
    src = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
    names = sorted(set(re.findall(r"\b(rnnt_[a-z_0-9]+)\s*\(", src)))
    assert names == sorted(enc.EXPORTED)
    lib = enc._library()
    for name in names:
        assert hasattr(lib, name), name


def call(fn, defaults, over):
    """fn on `defaults` (name -> value, in order) with some replaced."""
    args = dict(defaults)
    for k, v in over.items():
        assert k in args, k
        args[k] = v
    return fn(*args.values())


def test_norm_refusals(enc):
    lib, S = enc._library(), enc.NormShape
    ok = S(2, 3, 40, 1)
    fwd = {"x": FAKE, "residual": FAKE, "shape": ok, "lens": FAKE, "weight": FAKE, "eps": 0.0, "y": FAKE, "sum": FAKE,
           "stream": None}
    q8 = {"x": FAKE, "residual": FAKE, "shape": ok, "lens": FAKE, "weight": FAKE, "eps": 0.0, "q": FAKE, "pitch": 48,
          "scale": FAKE, "sum": FAKE, "stream": None}
    need = lib.rnnt_rms_norm_grad_workspace_bytes(ok)
    assert need > 0 and need % 256 == 0
    bwd = {"x": FAKE, "residual": FAKE, "shape": ok, "lens": FAKE, "weight": FAKE, "eps": 0.0, "dy": FAKE, "dsum": FAKE, "dx": FAKE, "dw": FAKE,
           "ws": FAKE, "bytes": need - 1, "stream": None}
    calls = ((lib.rnnt_rms_norm, fwd), (lib.rnnt_rms_norm8, q8), (lib.rnnt_rms_norm_grad, bwd))
    for shape, want in ((S(0, 3, 40, 1), 2), (S(2, -1, 40, 1), 2), (S(2, 3, 0, 1), 2), (S(2, 3, 40, 3), 4),
                        (S(2, 3, 32769, 1), 9), (S(2, 3, 16385, 0), 9), (S(1, 1 << 24, 40, 1), 9), (S(1, 1, 2**31 - 1, 1), 9)):
        for fn, args in calls:
            assert call(fn, args, {"shape": shape}) == want
        assert lib.rnnt_rms_norm_grad_workspace_bytes(shape) == 0
    for fn, args in calls:
        for eps in (-1.0, float("nan"), float("inf")):
            assert call(fn, args, {"eps": eps}) == 5
        assert call(fn, args, {"weight": None}) == 1 and call(fn, args, {"weight": FAKE + 1}) == 7
    for over, want in (({"x": None}, 1), ({"y": None}, 1), ({"sum": None}, 1), ({"x": FAKE + 1}, 7), ({"y": FAKE + 1}, 7),
                       ({"residual": FAKE + 1}, 7), ({"sum": FAKE + 1}, 7)):
        assert call(lib.rnnt_rms_norm, fwd, over) == want
    for over, want in (({"q": None}, 1), ({"scale": None}, 1), ({"q": FAKE + 8}, 7), ({"pitch": 40}, 7), ({"pitch": 32}, 7),
                       ({"scale": FAKE + 2}, 7), ({"sum": None}, 1)):
        assert call(lib.rnnt_rms_norm8, q8, over) == want
    for over, want in (({}, 6), ({"x": None}, 1), ({"dy": None}, 1), ({"dx": None}, 1), ({"dw": None}, 1), ({"dsum": None}, 6),
                       ({"residual": None}, 6), ({"x": FAKE + 1}, 7), ({"residual": FAKE + 1}, 7),
                       ({"dy": FAKE + 1}, 7), ({"dsum": FAKE + 1}, 7), ({"dw": FAKE + 1}, 7), ({"ws": FAKE + 16, "bytes": need}, 7)):
        assert call(lib.rnnt_rms_norm_grad, bwd, over) == want
    assert call(lib.rnnt_rms_norm, fwd, {"shape": S(2, 0, 40, 1), "x": None, "y": None}) == 0
    rows = {"x": FAKE, "rows": 3, "D": 40, "dtype": 1, "q": FAKE, "pitch": 48, "scale": FAKE, "stream": None}
    for over, want in (({"rows": -1}, 2), ({"D": 0}, 2), ({"dtype": 3}, 4), ({"rows": 1 << 24}, 9), ({"D": 32769, "pitch": 1 << 16}, 9),
                       ({"x": None}, 1), ({"q": None}, 1), ({"scale": None}, 1), ({"x": FAKE + 1}, 7), ({"q": FAKE + 8}, 7),
                       ({"pitch": 40}, 7), ({"pitch": 32}, 7), ({"scale": FAKE + 2}, 7), ({"rows": 0, "x": None}, 0)):
        assert call(lib.rnnt_quantize_rows, rows, over) == want


def test_linear8_refusals(enc):
    lib, S = enc._library(), enc.Linear8Shape
    ok = S(5, 7, 40, 1, 48, 48)
    fwd = {"x": FAKE, "xs": FAKE, "w": FAKE, "ws": FAKE, "shape": ok, "bias": FAKE, "y": FAKE, "stream": None}
    need = lib.rnnt_linear8_dynamic_workspace_bytes(S(3000, 3000, 4000, 1, 0, 4000))
    assert need > 0 and need % 256 == 0
    dyn = {"x": FAKE, "w": FAKE, "ws": FAKE, "shape": S(3000, 3000, 4000, 1, 0, 4000), "bias": FAKE, "y": FAKE, "work": FAKE,
           "bytes": need - 1, "stream": None}
    for shape, want in ((S(-1, 7, 40, 1, 48, 48), 2), (S(5, 0, 40, 1, 48, 48), 2), (S(5, 7, 0, 1, 48, 48), 2),
                        (S(5, 7, 40, 1, 48, 32), 2), (S(5, 7, 40, 3, 48, 48), 4), (S(5, 7, 40, 1, 48, 40), 7),
                        (S(1 << 24, 7, 40, 1, 48, 48), 9), (S(5, (1 << 21) + 1, 40, 1, 48, 48), 9), (S(5, 7, 1 << 17, 1, 1 << 17, 1 << 17), 9),
                        (S(5, 7, 40, 1, 48, 1 << 20), 9), (S(16777000, 2097000, 40, 1, 48, 48), 9)):
        assert call(lib.rnnt_linear8, fwd, {"shape": shape}) == want
        assert call(lib.rnnt_linear8_dynamic, dyn, {"shape": shape}) == want
        assert lib.rnnt_linear8_dynamic_workspace_bytes(shape) == 0
    for shape, want in ((S(5, 7, 40, 1, 32, 48), 2), (S(5, 7, 40, 1, 40, 48), 7), (S(5, 7, 40, 1, 1 << 20, 48), 9)):
        assert call(lib.rnnt_linear8, fwd, {"shape": shape}) == want
    for shape in (S(5, 7, 32769, 1, 0, 40000), S(5, 7, 16385, 0, 0, 40000)):
        assert call(lib.rnnt_linear8_dynamic, dyn, {"shape": shape}) == 9
    both = [({"x": None}, 1), ({"w": None}, 1), ({"ws": None}, 1), ({"y": None}, 1), ({"w": FAKE + 8}, 7), ({"ws": FAKE + 2}, 7),
            ({"bias": FAKE + 1}, 7), ({"y": FAKE + 1}, 7)]
    for over, want in both + [({"xs": None}, 1), ({"x": FAKE + 8}, 7), ({"xs": FAKE + 2}, 7)]:
        assert call(lib.rnnt_linear8, fwd, over) == want
    for over, want in both + [({}, 6), ({"x": FAKE + 1}, 7), ({"work": FAKE + 16, "bytes": need}, 7)]:
        assert call(lib.rnnt_linear8_dynamic, dyn, over) == want
    assert call(lib.rnnt_linear8, fwd, {"shape": S(0, 7, 40, 1, 48, 48), "x": None, "y": None}) == 0


def test_rotary_refusals(enc):
    lib, S = enc._library(), enc.RotaryShape
    ok = (2, 3, 4, 16, 8, 0, 1, 192, 64, 16)
    fwd = {"x": FAKE, "shape": S(*ok), "freq": FAKE, "start": FAKE, "lens": FAKE, "inverse": 0, "y": FAKE, "stream": None}
    for i, v, want in ((0, 0, 2), (1, -1, 2), (2, 0, 2), (3, 0, 2), (4, 0, 2), (4, 7, 2), (4, 18, 2), (7, -1, 2), (8, -1, 2), (9, -1, 2),
                       (6, 5, 4), (2, 5000, 9), (1, 1 << 23, 9)):
        shape = list(ok)
        shape[i] = v
        assert call(lib.rnnt_rotary, fwd, {"shape": S(*shape)}) == want, (i, v)
    assert call(lib.rnnt_rotary, fwd, {"shape": S(1, 1, 1, 2048, 1026, 0, 1, 0, 0, 0)}) == 9
    for over, want in (({"x": None}, 1), ({"freq": None}, 1), ({"y": None}, 1), ({"x": FAKE + 1}, 7), ({"y": FAKE + 1}, 7),
                       ({"freq": FAKE + 4}, 7)):
        assert call(lib.rnnt_rotary, fwd, over) == want
    assert call(lib.rnnt_rotary, fwd, {"shape": S(2, 0, *ok[2:]), "x": None, "y": None}) == 0


ATTENTION = {"B": 2, "L": 3, "Hq": 4, "Hkv": 2, "D": 64, "page": 16, "table": 300, "num_pages": 900, "causal": 1, "left": -1,
             "dtype": 1, **{"%s_%s" % (t, d): s for t, h in (("q", 4), ("k", 2), ("v", 2)) for d, s in (("b", 3 * h * 64), ("t", h * 64), ("h", 64))}}


def test_attention_refusals(enc):
    lib = enc._library()

    def S(**over):
        assert not set(over) - set(ATTENTION)
        return enc.AttentionShape(*{**ATTENTION, **over}.values())
    ok = S()
    need = lib.rnnt_cached_attention_workspace_bytes(ok)
    assert need > 0 and need % 256 == 0  # few tiles over a long table: shared out among blocks
    fwd = {"q": FAKE, "k": FAKE, "v": FAKE, "shape": ok, "lens": FAKE, "cached": FAKE, "pages": FAKE, "kc": FAKE, "vc": FAKE,
           "scale": 0.5, "out": FAKE, "ws": FAKE, "bytes": need - 1, "stream": None}
    for over, want in ((dict(B=0), 2), (dict(L=-1), 2), (dict(Hq=0), 2), (dict(Hkv=0), 2), (dict(D=0), 2), (dict(page=0), 2),
                       (dict(table=0), 2), (dict(num_pages=0), 2), (dict(Hq=3), 2), (dict(q_b=-64), 2), (dict(v_h=-64), 2),
                       (dict(dtype=3), 4), (dict(q_t=68), 7), (dict(k_b=4), 7), (dict(v_h=60), 7), (dict(D=60), 9), (dict(D=264), 9),
                       (dict(page=12), 9), (dict(page=2048), 9), (dict(num_pages=1 << 26), 9), (dict(table=1 << 26), 9),
                       (dict(L=1 << 29), 9), (dict(B=1 << 23), 9)):
        assert call(lib.rnnt_cached_attention, fwd, {"shape": S(**over)}) == want, over
        assert lib.rnnt_cached_attention_workspace_bytes(S(**over)) == 0
    for over, want in (({}, 6), ({"q": None}, 1), ({"k": None}, 1), ({"v": None}, 1), ({"cached": None}, 1), ({"pages": None}, 1),
                       ({"kc": None}, 1), ({"vc": None}, 1), ({"out": None}, 1), ({"scale": float("nan")}, 5), ({"scale": float("inf")}, 5),
                       ({"q": FAKE + 8}, 7), ({"k": FAKE + 8}, 7), ({"v": FAKE + 8}, 7), ({"kc": FAKE + 8}, 7), ({"vc": FAKE + 8}, 7),
                       ({"out": FAKE + 1}, 7), ({"ws": FAKE + 16, "bytes": need}, 7)):
        assert call(lib.rnnt_cached_attention, fwd, over) == want, over
    assert call(lib.rnnt_cached_attention, fwd, {"shape": S(L=0), "q": None, "out": None}) == 0


PAGES_PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "rnnt_pages.h"
using namespace rnnt;
int main() {
  // a table between guards that name no page: a read beside it would be seen
  for (int shift = 0; shift < 4; ++shift) {
    std::vector<int32_t> heap = {3, -1, 9, 8, 2147483647, -2147483647 - 1};
    PageTable t{heap.data(), static_cast<int32_t>(heap.size()), 9, shift};
    for (int64_t pos = -70000; pos < 70000; ++pos) {
      const int64_t i = pos >> shift;
      const int32_t want = pos < 0 || i >= 6 || heap[i] < 0 || heap[i] >= 9 ? -1 : heap[i];
      if (t.page_of(static_cast<int32_t>(pos)) != want) return 1;
    }
    for (int32_t pos : {2147483647, -2147483647 - 1})
      if (t.page_of(pos) != -1) return 2;
    for (int id = 0; id < 9; ++id)
      for (int h = 0; h < 3; ++h)
        for (int pos = 0; pos < 64; ++pos)
          if (cache_row(id, 3, h, pos, shift) != static_cast<uint32_t>((id * 3 + h) * (1 << shift) + pos % (1 << shift))) return 3;
  }
  if (cache_row(2097151, 64, 63, 15, 4) != 2147483647u) return 4;
  const int32_t far[] = {-2147483647 - 1, -1, 0, 1, 2, 5, 6, 7, 2147483647};
  for (int32_t n : far)
    for (int32_t c : far)
      if (lengths_fit(n, 5, c, 7) != (n >= 0 && n <= 5 && c >= 0 && static_cast<int64_t>(n) + c <= 7)) return 5;
  for (int left = -1; left < 9; ++left)
    for (int causal = 0; causal < 2; ++causal)
      for (int pos = 0; pos < 12; ++pos) {
        const Seen s(pos, 12, causal, left);
        for (int key = 0; key < 14; ++key) {
          const bool want = key < 12 && (!causal || key <= pos) && (left < 0 || key >= pos - left);
          if (s.holds(key) != want) return 6;
        }
      }
  if (Seen(5, 9, true, 2147483647).lo != 0) return 7;
  std::puts("fine");
  return 0;
}
"""


def test_arithmetic_of_pages_sanitized(tmp_path):
    """csrc/rnnt_pages.h on the host, under the address and undefined-behaviour sanitizers."""
    src, exe = tmp_path / "pages.cpp", tmp_path / "pages"
    src.write_text(PAGES_PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=" + "address,undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2303_10384_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True)
    assert got.returncode == 0 and got.stdout == "fine\n", (got.returncode, got.stderr)


def test_rotary_divisions():
    """The kernel divides item numbers below 2^16 by up to 2^16 through the high word of a product with 2^32 / d + 1."""
    for d in itertools.chain(range(2, 700), (1 << k for k in range(10, 17)), (65535, 65521, 43691)):
        m = (1 << 32) // d + 1
        for n in itertools.chain(range(0, 1 << 16, 251), (k * d + j for k in range(0, (1 << 16) // d, max(1, (1 << 16) // d // 40)) for j in (-1, 0, 1))):
            if 0 <= n < 1 << 16:
                assert n * m >> 32 == n // d


def test_binding_refuses_cpu_tensors(enc):
    import paper_2303_10384_amd as rnnt
    x = torch.zeros(2, 3, 16)
    w8 = rnnt.Rows8(torch.zeros(5, 16, dtype=torch.int8), torch.zeros(5))
    heads = x.view(2, 3, 2, 8)
    for call_it in (lambda: rnnt.rms_norm(x, x[0, 0]), lambda: rnnt.rms_norm8(x, x[0, 0]), lambda: rnnt.quantize_rows(x),
                    lambda: rnnt.linear8(x, w8), lambda: rnnt.rotary(heads, torch.zeros(2, dtype=torch.float64)),
                    lambda: rnnt.cached_attention(heads, heads, heads, heads, heads, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call_it()
    with pytest.raises(TypeError, match="tensor"):
        rnnt.rms_norm([1.0], x)
    with pytest.raises(TypeError, match="Rows8"):
        rnnt.linear8(x, (w8.values, w8.scale))


def test_rotary_frequencies(enc):
    import math
    f = enc.rotary_frequencies(8, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(enc.rotary_frequencies(8, stretch=4.0, device="cpu"), f / 4)
    # 1000 trained positions: 159, 15.9, 1.59 and 0.159 turns
    g = enc.rotary_frequencies(8, stretch=4.0, trained=1000, slow=1.0, fast=32.0, device="cpu")
    turns = 1000 * f / (2 * math.pi)
    keep = torch.tensor([1.0, float(turns[1] - 1) / 31, float(turns[2] - 1) / 31, 0.0], dtype=torch.float64)
    assert torch.allclose(g, f * (keep + (1 - keep) / 4), rtol=1e-14)
    assert torch.equal(enc.rotary_frequencies(8, trained=1000, device="cpu"), f)
    for bad in (dict(dim=0), dict(dim=3), dict(dim=4, base=0.0), dict(dim=4, stretch=-1.0), dict(dim=4, slow=2.0, fast=2.0)):
        with pytest.raises(ValueError):
            enc.rotary_frequencies(device="cpu", **bad)


def test_plain_forms_against_their_float64_results():
    """perf/more_operators.py on the CPU: its plain forms at half-step tolerances of their types."""
    import random
    from perf import more_operators as O
    rng = random.Random(11)
    cap = {"B": 3, "L": 40, "M": 70, "N": 50, "K": 300, "cached": 200}
    for _ in range(24):
        case = {k: min(v, cap[k]) if k in cap else v for k, v in O.draw(rng).items()}
        got, want = O.run(O.prepare(case, 3)), O.exact(case, 3)
        got, want = (v if isinstance(v, tuple) else (v,) for v in (got, want))
        assert len(got) == len(want)
        for g, w in zip(got, want):
            step = torch.finfo(g.dtype).eps / 2
            # each element's own rounding, and float32 arithmetic on values of the tensor's size; 8 bits: an integer more
            # or less where float32 and float64 lie on either side of a half
            off = 1.01 / 127 if case["mode"] == "infer8" else 2.0 ** -17
            assert g.shape == w.shape
            assert bool(((g.double() - w).abs() <= step * w.abs() + off * w.abs().max() + 1e-30).all()), case


# ---------------------------------------------------------------- the binding's calls, the library's stubbed

@pytest.fixture
def calls(enc, monkeypatch):
    """The entry points on CPU tensors: every library call is recorded as (name, arguments) and does nothing."""
    from paper_2303_10384_amd import binding
    made = []
    monkeypatch.setattr(enc, "_plans", {})  # what checks that are none find is not kept
    monkeypatch.setattr(enc, "_check", lambda *args, **kw: None)
    monkeypatch.setattr(enc, "_call", lambda fn, device, *args: made.append((fn.__name__, args)))
    monkeypatch.setattr(binding, "_capturing", lambda device: False)
    return made


def test_strides_of_views(enc, calls):
    import paper_2303_10384_amd as rnnt
    B, L, H, D = 2, 3, 4, 8
    both = torch.randn(B, L, 3, H, D, dtype=torch.float16)
    q, k, v = both.unbind(2)
    cache = torch.zeros(6, H, 16, D, dtype=torch.float16)
    pages, cached = torch.zeros(B, 3, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    rnnt.cached_attention(q, k, v, cache, cache.clone(), pages, cached, left=7, causal=False)
    s = calls[-1][1][3]
    assert (s.q_stride_b, s.k_stride_t, s.v_stride_h) == (L * 3 * H * D, 3 * H * D, D) and (s.left, s.causal) == (7, 0)
    # a dimension of one element names any stride
    rnnt.cached_attention(*(t[:, :1].as_strided((B, 1, H, D), (t.stride(0), 3, D, 1)) for t in (q, k, v)), cache, cache.clone(), pages, cached)
    s = calls[-1][1][3]
    assert s.q_stride_t == s.k_stride_t == 0 and s.left == -1
    freq = torch.zeros(3, dtype=torch.float64)
    x = q.detach().requires_grad_(True)
    y = rnnt.rotary(x, freq)
    torch.autograd.grad(y, x, torch.ones_like(y).transpose(1, 2).contiguous().transpose(1, 2))
    (_, fwd), (_, bwd) = calls[-2:]
    assert fwd[1].stride_t == 3 * H * D and fwd[5] == 0 and fwd[1].R == 6
    assert (bwd[1].stride_t, bwd[1].stride_h) == (D, L * D) and bwd[5] == 1


def test_sizes_past_32_bits_are_refused(enc, calls):
    import paper_2303_10384_amd as rnnt
    wide = (1 << 32) + 16
    meta = lambda *s, **kw: torch.empty(s, device="meta", **kw)  # noqa: E731
    i32, i8 = {"dtype": torch.int32}, {"dtype": torch.int8}
    w8 = rnnt.Rows8(meta(5, 16, **i8), meta(5))
    for call_it in (lambda: rnnt.rms_norm(meta(wide, 4), meta(4)), lambda: rnnt.rms_norm(meta(1, wide), meta(wide)),
                    lambda: rnnt.rms_norm8(meta(1, wide, 4), meta(4), None, meta(1, **i32)),
                    lambda: rnnt.quantize_rows(meta(1, wide)), lambda: rnnt.linear8(meta(wide, 16), w8),
                    lambda: rnnt.linear8(meta(1, wide), rnnt.Rows8(meta(5, wide, **i8), meta(5))),
                    lambda: rnnt.rotary(meta(1, wide, 1, 8), meta(4, dtype=torch.float64)),
                    lambda: rnnt.cached_attention(*[meta(1, wide, 1, 8)] * 3, *[meta(1, 1, 16, 8)] * 2, meta(1, 1, **i32), meta(1, **i32))):
        with pytest.raises(rnnt.RNNTError, match="UNSUPPORTED"):
            call_it()
    assert not calls


def test_gradients_past_a_launch_and_forward_mode(enc, calls):
    import torch.autograd.forward_ad as fw
    import paper_2303_10384_amd as rnnt
    x, w = torch.randn(2, 3, 16), torch.randn(16)
    heads, freq = x.view(2, 3, 2, 8), torch.zeros(2, dtype=torch.float64)
    w8 = rnnt.Rows8(torch.zeros(5, 16, dtype=torch.int8), torch.zeros(5))
    cache, pages, cached = torch.zeros(6, 2, 16, 8), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    attend = lambda q: rnnt.cached_attention(q, heads, heads, cache, cache.clone(), pages, cached)  # noqa: E731
    with fw.dual_level():
        dual = lambda t, grad=False: fw.make_dual(t.clone().requires_grad_(grad), torch.ones_like(t))  # noqa: E731
        for call_it in (lambda: rnnt.rms_norm(dual(x), w), lambda: rnnt.rms_norm(x, dual(w, True)), lambda: rnnt.rms_norm(x, w, dual(x)),
                        lambda: rnnt.rms_norm8(dual(x), w), lambda: rnnt.quantize_rows(dual(x)), lambda: rnnt.linear8(dual(x), w8),
                        lambda: rnnt.rotary(dual(heads), freq), lambda: attend(dual(heads))):
            with pytest.raises(NotImplementedError), torch.no_grad():
                call_it()
        n = len(calls)
        rnnt.linear8(x, w8)  # no tangent: as ever
        assert len(calls) == n + 1
    for call_it in (lambda t: rnnt.rms_norm8(t, w), rnnt.quantize_rows, lambda t: rnnt.linear8(t, w8), lambda t: attend(t.view(2, 3, 2, 8))):
        leaf = x.clone().requires_grad_(True)
        n = len(calls)
        with pytest.raises(RuntimeError, match="no gradient"):
            call_it(leaf)
        assert len(calls) == n
        with torch.no_grad():
            call_it(leaf)
        assert len(calls) == n + 1


def test_checks_are_made_again_for_other_tensors(enc, monkeypatch):
    """What the checks of a call found holds for tensors of its sizes, strides, types and GPU alone."""
    import paper_2303_10384_amd as rnnt
    from paper_2303_10384_amd import binding
    made = []
    monkeypatch.setattr(enc, "_plans", {})
    monkeypatch.setattr(enc, "_call", lambda fn, device, *args: made.append((fn.__name__, args)))
    monkeypatch.setattr(binding, "_capturing", lambda device: False)
    checks = []
    monkeypatch.setattr(enc, "_check", lambda name, t, *args, **kw: checks.append(name))
    x, w = torch.randn(4, 32), torch.randn(32)
    for t, again in ((x, True), (x.clone(), False), (torch.randn(5, 32), True), (torch.randn(32, 4).t(), True), (x.half(), True),
                     (x.clone(), False), (torch.randn(8, 32)[::2], True)):
        n = len(checks)
        rnnt.rms_norm(t, w)
        assert (len(checks) > n) == again
    w8 = rnnt.Rows8(torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5))
    odd = torch.zeros(5 * 32, dtype=torch.int8).as_strided((5, 20), (32, 1))
    short = torch.zeros(4 * 32 + 20, dtype=torch.int8).as_strided((5, 20), (32, 1))  # the last row ends inside 16 bytes
    rnnt.linear8(x, w8)
    rnnt.linear8(x[:, :20].contiguous(), rnnt.Rows8(odd, torch.zeros(5)))
    with pytest.raises(ValueError, match="pieces"):
        rnnt.linear8(x[:, :20].contiguous(), rnnt.Rows8(short, torch.zeros(5)))
    with pytest.raises(ValueError, match="x must be"):
        rnnt.linear8(x[:, :20].contiguous(), w8)
    for _ in range(2):
        with pytest.raises(TypeError, match="dtype"):
            rnnt.linear8(x, w8, dtype=torch.float16)
    for i in range(1030):  # and not without end
        rnnt.rms_norm(torch.empty(i + 1, 2), w[:2])
    assert len(enc._plans) <= 1024


def test_norm_gradient_of_tensors_saved_elsewhere(enc, calls):
    """Hooks on saved tensors may give any layout back: the gradient's call takes dense ones."""
    import paper_2303_10384_amd as rnnt
    x, w, r = torch.randn(2, 3, 16, requires_grad=True), torch.randn(16, requires_grad=True), torch.randn(2, 3, 16)
    for residual in (None, r):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.transpose(0, -1).contiguous().transpose(0, -1)):
            got = rnnt.rms_norm(x, w, residual)
            y = got if residual is None else got[0]
            torch.autograd.grad(y, (x, w), torch.ones_like(y).transpose(0, 1).contiguous().transpose(0, 1))
        name, bwd = calls[-1]
        assert name == "rnnt_rms_norm_grad" and bwd[7] is None and bwd[6] is not None and (bwd[1] is None) == (residual is None)


def test_autograd_sees_the_caches_written(enc, calls):
    """A tensor that shares memory with a cache and was saved for a backward pass is refused there after a call."""
    import paper_2303_10384_amd as rnnt
    pool = torch.zeros(2, 6, 2, 16, 8)
    pages, cached = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    q, k, v = torch.randn(2, 3, 4, 8), torch.randn(2, 3, 2, 8), torch.randn(2, 3, 2, 8)
    attend = lambda *caches: rnnt.cached_attention(q, k, v, *caches, pages, cached)  # noqa: E731
    for saved in (pool[0], pool[1], pool):
        leaf = torch.ones_like(saved, requires_grad=True)
        y = (leaf * saved).sum()
        attend(pool[0], pool[1])
        with pytest.raises(RuntimeError, match="inplace"):
            y.backward()
    leaf, apart = torch.ones_like(q, requires_grad=True), torch.zeros(2, 6, 2, 16, 8)
    y = (leaf * q).sum()  # the call's inputs are as they were
    attend(apart[0], apart[1])
    y.backward()
    versions = [t._version for t in (q, k, v, pages, cached)]
    with torch.inference_mode():  # caches without a counter
        made = torch.zeros(2, 6, 2, 16, 8)
        attend(made[0], made[1])
    assert versions == [t._version for t in (q, k, v, pages, cached)]


def test_linear8_limit_on_tiles(enc):
    """2^23 - 1 tiles of 128 x 128 results are taken (and end at the next check), 2^23 are not."""
    lib, S = enc._library(), enc.Linear8Shape
    for M, N, want in ((511 * 128, 1 << 21, 1), (511 * 128 + 1, 1 << 21, 9), (8191 * 128, 1024 * 128, 1), (8191 * 128 + 1, 1024 * 128, 9),
                       ((1 << 23) - 128, 127 * 128 + 1, 1), ((1 << 24) - 1, 63 * 128, 1), ((1 << 24) - 1, 64 * 128, 9)):
        shape = S(M, N, 40, 1, 48, 48)
        assert lib.rnnt_linear8(None, FAKE, FAKE, FAKE, shape, None, FAKE, None) == want, (M, N)
        assert lib.rnnt_linear8_dynamic(None, FAKE, FAKE, shape, None, FAKE, None, 0, None) == want, (M, N)


def test_attention_scale_past_float32_in_powers_of_two(enc):
    """The kernels take scores in powers of two: a scale whose product with log2 e is no float32 is refused, the largest one
    below goes on to the next check."""
    lib = enc._library()
    ok = enc.AttentionShape(*ATTENTION.values())
    fwd = {"q": FAKE, "k": FAKE, "v": FAKE, "shape": ok, "lens": FAKE, "cached": FAKE, "pages": FAKE, "kc": FAKE, "vc": FAKE,
           "scale": 0.5, "out": None, "ws": None, "bytes": 0, "stream": None}
    for scale, want in ((2.3586e38, 1), (-2.3586e38, 1), (2.3587e38, 5), (-2.3587e38, 5), (3.4e38, 5)):
        assert call(lib.rnnt_cached_attention, fwd, {"scale": scale}) == want, scale
