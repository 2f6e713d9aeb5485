"""The encoder's operators on the GPU against the float64 reference: values, gradients, lengths,
strides, masks, pages, streams, captured graphs, and the operators chained as a layer.

Tolerances.  HALF[dtype] is the half step of the stored type, relative to the value; float32
arithmetic inside is off by ONE = 2^-24 of a product, sum or conversion, the reciprocal square
root and the exponential by 2^-23 and 2^-22."""
import sys

import numpy as np
import pytest

from oracle import encoder_ref as R
from test_gpu_network import DTYPES, HALF, ONE, TINY, close, ints, rounded, td
from test_gpu_parity import pkg, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def announce(request):
    sys.__stderr__.write("\n[gpu-test] %s\n" % request.node.nodeid)
    sys.__stderr__.flush()
    yield


def rng_of(seed):
    return np.random.Generator(np.random.PCG64(seed))


def some_lengths(rng, kind, B, L):
    return None if kind is None else rng.integers(0, L + 1, size=B) if kind == "any" else np.full(B, L if kind == "full" else 0)


# ---------------------------------------------------------------- root-mean-square norm

NORM = [  # B, L, D, lengths, residual
    (1, 1, 1, None, False), (2, 3, 7, "any", True), (16, 1, 640, None, True), (3, 5, 8, "any", False),
    (4, 33, 64, "any", True), (2, 9, 65, "full", False), (5, 2, 129, "any", True), (3, 4, 257, "any", True),
    (2, 3, 512, "zero", True), (2, 5, 635, "any", True), (1, 7, 1024, None, False), (2, 2, 1025, "any", True),
    (2, 3, 2048, "any", False), (2, 2, 2051, "any", True), (1, 3, 8192, None, True), (1, 2, 9001, "any", False),
    (2, 0, 16, "any", True), (64, 40, 33, "any", True), (7, 300, 40, "any", False), (1, 2, 16384, None, True)]


def norm_case(torch, case, dtype, seed):  # noqa: F811
    B, L, D, lengths, with_residual = case
    rng = rng_of(seed)
    lens = some_lengths(rng, lengths, B, L)
    x, xd = rounded(torch, rng.standard_normal((B, L, D)), dtype)
    w, wd = rounded(torch, 1.0 + 0.3 * rng.standard_normal(D), dtype)
    r, rd = rounded(torch, 2.0 * rng.standard_normal((B, L, D)), dtype) if with_residual else (None, None)
    if lens is not None:
        for b in range(B):  # never used
            x[b, lens[b]:] = float("nan")
            if r is not None:
                r[b, lens[b]:] = float("inf")
    return rng, x, xd, w, wd, r, rd, lens


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", NORM)
def test_norm(torch, pkg, case, dtype):  # noqa: F811
    rng, x, xd, w, wd, r, rd, lens = norm_case(torch, case, dtype, 1)
    leaves = [t.requires_grad_(True) for t in (x, w, r) if t is not None]
    got = pkg.rms_norm(x, w, r, ints(torch, lens), eps=1e-3)
    y, total = got if r is not None else (got, None)
    want, t = R.rms_norm(xd, wd, rd, lens, 1e-3)
    # a lane adds up at most 32 squares, then up to 10 steps join the lanes: 42 roundings, halved by the root;
    # the mean, eps, root, and two products; and t's own rounding
    arith = (42 / 2 + 8) * ONE
    close(y, want, (HALF[dtype] + arith) * np.abs(want) + TINY[dtype], "y")
    if r is not None:
        close(total, t, (HALF[dtype] + ONE) * np.abs(t) + TINY[dtype], "sum")
    dy, dyd = rounded(torch, rng.standard_normal(xd.shape), dtype)
    ds, dsd = rounded(torch, rng.standard_normal(xd.shape), dtype)
    if lens is not None:
        for b in range(x.shape[0]):
            dy[b, lens[b]:] = float("nan")
            ds[b, lens[b]:] = float("nan")
    ups = (dy, ds) if r is not None else (dy,)
    heads = (y, total) if r is not None else (y,)
    grads = torch.autograd.grad(heads, leaves, ups, retain_graph=True)
    dx, dw, size, dw_size = R.rms_norm_grad(t, wd, dyd, dsd if r is not None else None, lens, 1e-3)
    # sums of up to 42 roundings in the two sums, the square's half twice; a few products around them; t's own rounding
    close(grads[0], dx, HALF[dtype] * np.abs(dx) + 2 * 60 * ONE * size + TINY[dtype], "dx")
    n = x.shape[0] * x.shape[1]
    # a column: its rows in order within a block and the blocks' sums, at most n roundings; r and two products
    close(grads[1], dw, HALF[dtype] * np.abs(dw) + (n + 40) * ONE * dw_size + TINY[dtype], "dw")
    if r is not None:
        assert torch.equal(grads[0], grads[2])
    again = torch.autograd.grad(heads, leaves, ups, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    if r is not None:  # only one of the results used
        only = torch.autograd.grad(total, leaves, ds, retain_graph=True)
        valid = np.ones(xd.shape[:2], bool) if lens is None else np.arange(xd.shape[1])[None] < lens[:, None]
        close(only[0], np.where(valid[..., None], dsd, 0.0), 0.0, "dsum alone")
        assert not bool(only[1].any())
        only = torch.autograd.grad(y, leaves, dy)
        dx, _, size, _ = R.rms_norm_grad(t, wd, dyd, None, lens, 1e-3)
        close(only[0], dx, HALF[dtype] * np.abs(dx) + 2 * 60 * ONE * size + TINY[dtype], "dy alone")
    with torch.no_grad():
        again = pkg.rms_norm(x, w, r, ints(torch, lens), eps=1e-3)
    assert torch.equal(again if r is None else again[0], y)


def test_norm_gradient_of_many_rows(torch, pkg):  # noqa: F811
    """More rows than a block's turn holds; whole numbers and a unit scale would not test the sums, so against float64."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for B, L, D in ((9, 4001, 96), (3, 20011, 40), (2, 3001, 2056)):
        x = torch.randn((B, L, D), device="cuda", generator=g).requires_grad_(True)
        w = torch.randn((D,), device="cuda", generator=g).requires_grad_(True)
        dy = torch.randn((B, L, D), device="cuda", generator=g)
        lens = torch.randint(0, L + 1, (B,), device="cuda", generator=g).to(torch.int32)
        dx, dw = torch.autograd.grad(pkg.rms_norm(x, w, None, lens), (x, w), dy)
        valid = (torch.arange(L, device="cuda")[None] < lens[:, None])[..., None]
        t = x.detach().double()
        r = 1 / (t.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt()
        d, unit = torch.where(valid, dy.double(), 0.0), t * r
        k = d * w.detach().double()
        want = r * (k - unit * (k * unit).mean(-1, keepdim=True))
        size = r * (k.abs() + unit.abs() * (k * unit).abs().mean(-1, keepdim=True))
        assert bool(((dx - want).abs() <= 120 * ONE * size + 1e-30).all())
        terms = d * unit
        assert bool(((dw - terms.sum((0, 1))).abs() <= (B * L / 64 + 100) * ONE * terms.abs().sum((0, 1))).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_bad_lengths_and_odd_values(torch, pkg, dtype):  # noqa: F811
    rng, x, xd, w, wd, r, rd, _ = norm_case(torch, (4, 3, 20, None, True), dtype, 5)
    lens = np.array([3, 4, -1, 2])
    x.requires_grad_(True)
    y, t = pkg.rms_norm(x, w, r, ints(torch, lens))
    want, total = R.rms_norm(xd, wd, rd, lens)
    close(y, want, (HALF[dtype] + 32 * ONE) * np.abs(want), "y")
    close(t, total, (HALF[dtype] + ONE) * np.abs(total), "sum")
    (dx,) = torch.autograd.grad(y, x, torch.ones_like(y))
    assert not bool(dx[1:3].any()) and bool(dx[0].any())
    rows, t8 = pkg.rms_norm8(x.detach(), w, r, ints(torch, lens))
    assert bool(rows.scale[1:3].isnan().all()) and not bool(rows.values[1:3].any()) and bool(t8[1:3].isnan().all())
    assert bool((rows.scale[3, 2:] == 0).all()) and bool((rows.scale[3, :2] > 0).all())
    odd = torch.ones((1, 3, 20), device="cuda", dtype=td(torch, dtype))
    odd[0, 0, 3], odd[0, 1, 4] = float("inf"), float("nan")
    y = pkg.rms_norm(odd, w)
    assert bool(y[0, 1].isnan().all()) and bool(y[0, 0, 3].isnan()) and bool((y[0, 0, :3] == 0).all()) and bool(y[0, 2].isfinite().all())
    rows = pkg.rms_norm8(odd, w)
    assert bool(rows.scale[0, :2].isnan().all()) and not bool(rows.values[0, :2].any()) and bool(rows.scale[0, 2] > 0)
    zero = torch.zeros((2, 20), device="cuda", dtype=td(torch, dtype))
    assert not bool(pkg.rms_norm(zero, w).any()) and not bool(pkg.rms_norm8(zero, w).scale.any())


# ---------------------------------------------------------------- rows in 8 bits

def check_rows8(rows, quotient, scale, arith, what):
    """quotients 127 v / max known to `arith` of themselves: their integers, which may be either neighbour of a half
    that lies within that, and the scales."""
    q = rows.values.cpu().numpy().astype(np.float64)
    assert q.shape == quotient.shape, what
    near = np.abs(np.abs(quotient - np.floor(quotient)) - 0.5) <= arith * 127
    assert np.array_equal(np.where(near, 0, q), np.where(near, 0, np.rint(quotient))), what
    assert np.all(np.abs(q - quotient) <= 0.5 + arith * 127), what
    close(rows.scale, scale, (arith + 4 * ONE) * scale, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", NORM)
def test_norm8(torch, pkg, case, dtype):  # noqa: F811
    _, x, xd, w, wd, r, rd, lens = norm_case(torch, case, dtype, 2)
    got = pkg.rms_norm8(x, w, r, ints(torch, lens), eps=1e-3)
    rows, total = got if r is not None else (got, None)
    want, t = R.rms_norm(xd, wd, rd, lens, 1e-3)
    quotient, scale = R.quantize_rows(want.reshape(-1, want.shape[-1]))
    # t, its product with the weight, and the quotient; the scale has the norm's 30 roundings besides
    check_rows8(pkg.Rows8(rows.values.reshape(-1, want.shape[-1]), rows.scale.reshape(-1)), quotient, scale, 32 * ONE, "rows")
    if r is not None:
        close(total, t, (HALF[dtype] + ONE) * np.abs(t) + TINY[dtype], "sum")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(1, 1), (3, 5), (7, 16), (5, 40), (33, 100), (4, 640), (2, 1025), (3, 2056), (2, 16384), (0, 8)])
def test_quantized_rows(torch, pkg, M, K, dtype):  # noqa: F811
    rng = rng_of(M + K)
    x, xd = rounded(torch, rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1)) * 3), dtype)
    rows = pkg.quantize_rows(x)
    quotient, scale = R.quantize_rows(xd)
    # values of 16 bits: the product with 127 is exact, and so is a quotient that is a half
    check_rows8(rows, quotient, scale, 0.0 if dtype != "f32" else 3 * ONE, "rows")
    assert rows.values.stride(0) % 16 == 0 or M < 2


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantized_halves_and_extremes(torch, pkg, dtype):  # noqa: F811
    """Every half of a row goes to the even side, at any power of two that the type holds; rows of zeros and odd values."""
    top = {"f32": 2.0 ** 120, "bf16": 2.0 ** 120, "f16": 2.0 ** 8}[dtype]
    low = {"f32": 2.0 ** -90, "bf16": 2.0 ** -90, "f16": 2.0 ** -15}[dtype]
    halves = np.concatenate([[127.0], np.arange(-64, 64) + 0.5, [63.0, -127.0]])
    for by in (1.0, top, low):
        x, xd = rounded(torch, halves[None] * by, dtype)
        assert np.array_equal(xd, halves[None] * by)
        rows = pkg.quantize_rows(x)
        assert np.array_equal(rows.values.cpu().numpy()[0], np.rint(halves)) and float(rows.scale[0]) == by
    x = torch.ones((6, 9), device="cuda", dtype=td(torch, dtype))
    x[0] = 0
    x[1, 8], x[2, 0], x[3, 4] = float("nan"), float("inf"), float("-inf")
    x[4] *= 2.0 ** -20  # not so small that it counts as nothing
    rows = pkg.quantize_rows(x)
    assert bool(rows.scale[1:4].isnan().all()) and not bool(rows.values[:4].any()) and float(rows.scale[0]) == 0
    assert bool((rows.values[4:] == 127).all())
    if dtype != "f16":
        tiny = torch.full((1, 3), 2.0 ** -101, device="cuda", dtype=td(torch, dtype))
        assert float(pkg.quantize_rows(tiny).scale[0]) == 0 and not bool(pkg.quantize_rows(tiny).values.any())


# ---------------------------------------------------------------- product in 8 bits

LINEAR = [  # M, K, N
    (1, 1, 1), (1, 16, 33), (3, 5, 7), (16, 640, 1025), (2, 100, 64), (17, 127, 130), (64, 128, 128), (65, 129, 257),
    (130, 48, 31), (200, 640, 96), (300, 321, 200), (129, 1000, 129), (40, 2048, 17), (257, 64, 1025), (33, 4096, 40),
    (0, 8, 4), (15, 2047, 1), (1100, 256, 160), (128, 16, 300), (513, 1040, 272),
    # past the form for few rows: rows held in registers, and rows too long for that
    (700, 127, 1000), (2100, 640, 300), (1500, 1024, 501), (4100, 5, 257), (33000, 130, 15), (2049, 768, 289), (1100, 1040, 1000),
    (2048, 1030, 523), (40, 3969, 70), (30, 5000, 33), (900, 516, 700), (20, 3420, 70)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_linear8(torch, pkg, M, K, N, dtype):  # noqa: F811
    rng = rng_of(M * 7 + K + N)
    pitch = -(-K // 16) * 16
    q, w = rng.integers(-128, 128, size=(M, K)), rng.integers(-128, 128, size=(N, K))

    def rows8(a, scale):
        # what lies between K and the pitch counts for nothing
        t = torch.full((len(a), pitch), 77, dtype=torch.int8, device="cuda")
        t[:, :K] = torch.from_numpy(a.astype(np.int8)).to("cuda")
        return pkg.Rows8(t[:, :K], torch.from_numpy(scale.astype(np.float32)).to("cuda"))
    qs, ws = (np.exp(rng.standard_normal(n)).astype(np.float32) / 127 for n in (M, N))
    bias, biasd = rounded(torch, 10 * rng.standard_normal(N), dtype)
    x8, w8 = rows8(q, qs), rows8(w, ws)
    for b, bd in ((bias, biasd), (None, None)):
        y = pkg.linear8(x8, w8, b, dtype=td(torch, dtype))
        want, size = R.linear8(q, qs, w, ws, bd)
        # the sum is exact; its conversion, two products with scales, the bias
        close(y, want, HALF[dtype] * np.abs(want) + 4 * ONE * size + TINY[dtype], "y")
    # rows in 16 or 32 bits, taken to 8 within the call: the same as in two calls
    x, _ = rounded(torch, rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1))), dtype)
    y = pkg.linear8(x, w8, bias)
    rows = pkg.quantize_rows(x)
    want, size = R.linear8(rows.values.cpu().numpy(), rows.scale.cpu().numpy().astype(np.float64), w, ws, biasd)
    close(y, want, HALF[dtype] * np.abs(want) + 4 * ONE * size + TINY[dtype], "y of rows")
    assert torch.equal(y, pkg.linear8(rows, w8, bias, dtype=td(torch, dtype)))


def test_linear8_largest_sums(torch, pkg):  # noqa: F811
    """The longest rows of the lowest values: 2^31 - 2^14, exactly."""
    K = (1 << 17) - 1
    x = torch.full((3, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    w = torch.full((5, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    y = pkg.linear8(pkg.Rows8(x, one(3)), pkg.Rows8(w, one(5)))
    assert bool((y == float(K * 128 * 128)).all())


def test_linear8_odd_rows(torch, pkg):  # noqa: F811
    """Rows that hold an infinity or NaN give NaN, zeros give the bias; leading dimensions and a strided view."""
    g = torch.Generator(device="cuda").manual_seed(1)
    w = pkg.quantize_rows(torch.randn((24, 40), device="cuda", generator=g))
    bias = torch.randn((24,), device="cuda", generator=g)
    x = torch.randn((3, 2, 40), device="cuda", generator=g)
    x[0, 1, 5], x[1, 0] = float("nan"), 0
    y = pkg.linear8(x, w, bias)
    assert bool(y[0, 1].isnan().all()) and torch.equal(y[1, 0], bias) and bool(y[2].isfinite().all())
    wide = torch.zeros((6, 96), dtype=torch.int8, device="cuda")
    rows = pkg.quantize_rows(x)
    wide[:, 16:56] = rows.values.reshape(6, 40)
    view = pkg.Rows8(wide[:, 16:56].view(3, 2, 40), rows.scale)
    assert torch.equal(pkg.linear8(view, w, bias).nan_to_num(7.0), y.nan_to_num(7.0))
    assert torch.equal(pkg.linear8(pkg.Rows8(wide[4, 16:56], rows.scale[2, 0]), w, bias), y[2, 0])


# ---------------------------------------------------------------- rotary positions

ROTARY = [  # B, L, H, D, R, lengths, start, layout
    (1, 1, 1, 2, 2, None, None, "dense"), (2, 5, 3, 8, 8, "any", "far", "dense"), (3, 4, 2, 64, 64, "any", "near", "thirds"),
    (2, 7, 4, 64, 32, "any", "far", "dense"), (1, 9, 2, 40, 6, None, "far", "heads first"), (4, 3, 5, 7, 4, "any", "near", "dense"),
    (2, 33, 16, 96, 96, "any", "far", "thirds"), (2, 3, 1, 130, 34, "zero", "near", "dense"), (2, 6, 2, 80, 22, "full", "far", "thirds"),
    (1, 1100, 2, 16, 16, None, "far", "dense"), (2, 0, 3, 8, 4, None, None, "dense"), (1, 3, 1, 1024, 1024, "any", "far", "dense"),
    (2, 2, 40, 24, 18, "any", "far", "heads first")]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", ROTARY)
def test_rotary(torch, pkg, case, interleaved, dtype):  # noqa: F811
    B, L, H, D, turned, lengths, far, layout = case
    rng = rng_of(B + L + H + D)
    if layout == "thirds":
        both, bothd = rounded(torch, rng.standard_normal((B, L, 3, H, D)), dtype)
        x, xd = both.clone()[:, :, 1], bothd[:, :, 1]
    else:
        x, xd = rounded(torch, rng.standard_normal((B, L, H, D)), dtype)
        if layout == "heads first":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
    lens = some_lengths(rng, lengths, B, L)
    start = None if far is None else rng.integers(0, 1000000 if far == "far" else 3, size=B)
    if lens is not None:
        for b in range(B):
            x[b, lens[b]:] = float("nan")
    freq = pkg.rotary_frequencies(turned, stretch=2.0, trained=500)
    fd = freq.cpu().numpy()
    x = x.detach().requires_grad_(True)
    y = pkg.rotary(x, freq, ints(torch, start), ints(torch, lens), interleaved=interleaved)
    want, size = R.rotary(xd, fd, start, lens, interleaved)
    # what is left of the angle is off by 2^-25 of a turn (2^-22.3), sine and cosine by 2^-23 besides; two products and a sum
    tol = HALF[dtype] * np.abs(want) + (2.0 ** -21 + 2 * ONE) * size + TINY[dtype] * (size > 0)
    close(y, want, tol, "y")
    dy, dyd = rounded(torch, rng.standard_normal(want.shape), dtype)
    if lens is not None:
        for b in range(B):
            dy[b, lens[b]:] = float("nan")
    (dx,) = torch.autograd.grad(y, x, dy, retain_graph=True)
    want, size = R.rotary(dyd, fd, start, lens, interleaved, -1.0)
    close(dx, want, HALF[dtype] * np.abs(want) + (2.0 ** -21 + 2 * ONE) * size + TINY[dtype] * (size > 0), "dx")
    strided = dy.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(torch.autograd.grad(y, x, strided)[0], dx)


def test_rotary_far_positions_and_bad_lengths(torch, pkg):  # noqa: F811
    """Positions up to the end of int32, and before 0: angles of 2^31 radians keep 2^-22 of one."""
    freq = pkg.rotary_frequencies(16)
    start = np.array([2**31 - 3, -5, 2**24 + 1, -2**31])
    x, xd = rounded(torch, rng_of(4).standard_normal((4, 2, 3, 16)), "f32")
    y = pkg.rotary(x, freq, ints(torch, start))
    want, size = R.rotary(xd, freq.cpu().numpy(), start)
    # three float64 roundings of an angle of 2^31, here and in the reference's angle, its sine and its cosine
    close(y, want, (2.0 ** -21 + 6 * 2.0 ** 31 * 2.0 ** -53 + 2 * ONE) * size, "y")
    y = pkg.rotary(x, freq, None, ints(torch, [2, 3, -1, 0]))
    assert bool(y[1:3].isnan().all()) and not bool(y[3].any()) and bool(y[0].isfinite().all())


# ---------------------------------------------------------------- attention over a paged cache

def attention_case(torch, B, L, Hq, Hkv, D, page, cached, lens, dtype, seed, layout="dense", spare=2, sigma=1.0):  # noqa: F811
    """Tensors of a call and their values; slots that hold no token are NaN, and so is what lies behind lens."""
    rng = rng_of(seed)
    cached = np.asarray(cached)
    width = max(1, -(-int(cached.max() + L) // page)) + spare
    P = B * width + 3
    pages = rng.permutation(P)[:B * width].reshape(B, width)
    shapes = ((B, L, Hq, D), (B, L, Hkv, D), (B, L, Hkv, D))
    if layout == "fused":
        both, bothd = rounded(torch, rng.standard_normal((B, L, (Hq + 2 * Hkv) * D)) * sigma, dtype)
        cut = [0, Hq * D, (Hq + Hkv) * D, (Hq + 2 * Hkv) * D]
        new = [both.clone()[:, :, a:b].unflatten(2, (-1, D)) for a, b in zip(cut, cut[1:])]
        newd = [bothd[:, :, a:b].reshape(B, L, -1, D) for a, b in zip(cut, cut[1:])]
    else:
        new, newd = zip(*(rounded(torch, rng.standard_normal(s) * sigma, dtype) for s in shapes))
        if layout == "heads first":
            new = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in new]
    caches, cachesd = zip(*(rounded(torch, rng.standard_normal((P, Hkv, page, D)) * sigma, dtype) for _ in range(2)))
    held = np.zeros((P, page), bool)
    for b in range(B):
        j = np.arange(cached[b])
        held[pages[b, j // page], j % page] = True
        if lens is not None:
            for t in new:
                t[b, lens[b]:] = float("nan")
    for t in caches:
        t[torch.from_numpy(~held).to("cuda")[:, None, :, None].expand(t.shape)] = float("nan")
        assert t.is_contiguous()
    for b in range(B):  # behind the tokens the table may hold anything
        used = -(-(int(cached[b]) + (L if lens is None else int(lens[b]))) // page)
        pages[b, used:] = [-1, P, 2**31 - 1, -2**31][b % 4]
    return list(new), list(newd), list(caches), list(cachesd), pages, held


def attention_tolerance(want, size, score_size, D, keys, v_max, dtype):
    """float32 sums over D in the scores (their sizes), the exponent's 2^-22, weights rounded as values are,
    sums over keys, the waves' and splits' joining; weights of float16 below 2^-14 are off by 2^-25."""
    ds = (D + 8) * ONE * score_size + 2.0 ** -21
    weights = 0.0 if dtype == "f32" else HALF[dtype]
    small = keys * 2.0 ** -25 * v_max if dtype == "f16" else 0.0
    return HALF[dtype] * np.abs(want) + (2 * ds + 2 * weights + (keys + 300) * ONE) * size + small + TINY[dtype]


def check_attention(torch, pkg, new, newd, caches, cachesd, pages, cached, lens, dtype, **kw):  # noqa: F811
    before = [c.clone() for c in caches]
    out = pkg.cached_attention(*new, *caches, ints(torch, pages), ints(torch, cached), ints(torch, lens), **kw)
    want, size, score_size, k_after, v_after = R.cached_attention(*newd, *cachesd, pages, cached, lens, **kw)
    keys = int(np.max(cached)) + newd[0].shape[1]
    v_max = max(np.abs(newd[2]).max(initial=0.0), np.abs(cachesd[1]).max())
    close(out, want, attention_tolerance(want, size, score_size, newd[0].shape[3], keys, v_max, dtype), "out")
    for got, was, after, at_first in zip(caches, before, (k_after, v_after), cachesd):
        # the rows of the new tokens, to the bit, and nothing else
        changed = np.any(after != at_first, axis=-1)
        close(got[torch.from_numpy(changed).to("cuda")], after[changed], 0.0, "cache")
        same = torch.from_numpy(~changed).to("cuda")
        assert torch.equal(got[same].nan_to_num(9.0), was[same].nan_to_num(9.0))
    return out


ATTENTION = [  # B, L, Hq, Hkv, D, page, cached, lens, layout, options
    (1, 1, 1, 1, 8, 1, [0], None, "dense", {}),
    (1, 1, 1, 1, 64, 16, [40], None, "dense", {}),
    (3, 1, 4, 4, 64, 16, [0, 16, 79], None, "fused", {}),
    (2, 1, 8, 2, 32, 8, [31, 64], [1, 0], "dense", {"left": 10}),
    (3, 5, 4, 2, 40, 4, [0, 7, 30], [5, 3, 0], "fused", {}),
    (2, 16, 2, 2, 64, 16, [33, 90], [16, 9], "fused", {"causal": False, "left": 20}),
    (2, 16, 2, 1, 128, 32, [50, 0], [16, 1], "heads first", {"causal": False}),
    (2, 9, 6, 2, 96, 8, [70, 13], None, "dense", {"left": 0}),
    (2, 7, 3, 1, 80, 64, [128, 63], [7, 6], "fused", {"left": 5}),
    (1, 3, 20, 1, 16, 2, [11], None, "dense", {}),
    (1, 2, 2, 1, 256, 16, [37], None, "dense", {}),
    (1, 3, 2, 2, 200, 1024, [5], None, "dense", {"causal": False}),
    (2, 40, 2, 1, 64, 16, [0, 21], [40, 33], "fused", {}),
    (1, 70, 1, 1, 24, 16, [10], None, "dense", {"left": 33}),
    (1, 130, 2, 2, 64, 32, [3], [129], "fused", {"causal": False, "left": 40}),
    (2, 150, 4, 1, 128, 16, [60, 0], [150, 77], "fused", {}),
    (2, 0, 2, 1, 64, 16, [5, 6], None, "dense", {}),
    (1, 1, 2, 1, 64, 16, [9], None, "dense", {"scale": 0.7}),
    (1, 4, 2, 1, 64, 16, [9], None, "dense", {"scale": 0.0}),
    (1, 6, 2, 1, 64, 16, [30], None, "dense", {"scale": -0.3})]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "-".join(map(str, c[:6])))
def test_attention(torch, pkg, case, dtype):  # noqa: F811
    B, L, Hq, Hkv, D, page, cached, lens, layout, options = case
    cached, lens = np.array(cached), None if lens is None else np.array(lens)
    new, newd, caches, cachesd, pages, _ = attention_case(torch, B, L, Hq, Hkv, D, page, cached, lens, dtype, B + L + D, layout)
    out = check_attention(torch, pkg, new, newd, caches, cachesd, pages, cached, lens, dtype, **options)
    assert torch.equal(out, pkg.cached_attention(*new, *caches, ints(torch, pages), ints(torch, cached), ints(torch, lens), **options))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L,G,causal", [(5, 1, True), (40, 2, True), (40, 2, False), (150, 1, True)])
def test_attention_large_scores_and_odd_values(torch, pkg, L, G, causal, dtype):  # noqa: F811
    """Scores of hundreds, whose maximum grows from key to key; an infinity and NaN among keys and values reach the
    queries that see them and no other."""
    cached = np.array([70, 33])
    new, newd, caches, cachesd, pages, _ = attention_case(torch, 2, L, 2 * G, 2, 64, 16, cached, None, dtype, L, sigma=3.0)
    options = {"causal": causal, "left": 50}
    v_max = max(np.abs(newd[2]).max(), np.abs(cachesd[1]).max())

    def near(b):
        # a step that holds odd values adds up weights that are not rounded first, in another order: the weights' and the
        # result's roundings on either side, and sums over up to 200 keys
        return 4 * HALF[dtype] * v_max + 400 * ONE * v_max
    check_attention(torch, pkg, new, newd, caches, cachesd, pages, cached, None, dtype, **options)
    with torch.no_grad():
        clean = pkg.cached_attention(*new, *caches, ints(torch, pages), ints(torch, cached), **options)
        spots = ((0, "v", 3, float("nan")), (1, "v", L - 2, float("inf")), (0, "k", L - 1, float("nan")))
        for b, what, t, value in spots:
            turned = [x.clone() for x in new]
            turned["qkv".index(what)][b, t, 1, 5] = value
            out = pkg.cached_attention(*turned, *[c.clone() for c in caches], ints(torch, pages), ints(torch, cached), **options)
            at = np.arange(L)
            sees = (t <= at if causal else np.ones(L, bool)) & (t >= at - 50)
            heads = np.arange(2 * G) // G == 1
            reach = np.zeros((2, L, 2 * G, 64), bool)
            reach[b] = (sees[:, None] & heads[None])[..., None] & ((np.arange(64) == 5) if what == "v" else True)
            reach = torch.from_numpy(reach).to("cuda")
            assert bool(((out - clean)[~reach].abs() <= near(b)).all()), (what, t)
            assert torch.equal(out[1 - b], clean[1 - b])
            assert not bool(out[reach].isfinite().any())
        # in the cache: token 60 of utterance 0, which the first queries see and the later ones do not
        old = [c.clone() for c in caches]
        old[1][int(pages[0, 60 // 16]), 0, 60 % 16, 7] = float("nan")
        out = pkg.cached_attention(*new, *old, ints(torch, pages), ints(torch, cached), **options)
        sees = 60 >= 70 + np.arange(L) - 50
        assert bool(out[0, torch.from_numpy(sees).to("cuda"), :G, 7].isnan().all())
        rest = torch.from_numpy(~sees).to("cuda")
        assert bool(((out - clean)[0, rest].abs() <= near(0)).all()) and torch.equal(out[1], clean[1])


def test_attention_bad_lengths_and_pages(torch, pkg):  # noqa: F811
    for L in (3, 40):
        cached = np.array([20, 20, 20, 20])
        new, newd, caches, cachesd, pages, held = attention_case(torch, 4, L, 2, 1, 64, 16, cached, None, "bf16", 9, spare=0)
        capacity = pages.shape[1] * 16
        for wrong, lens in (([20, -1, capacity - L + 1, 2**31 - 1], None), ([20] * 4, [1, L + 1, -1, -2**31])):
            mine = [c.clone() for c in caches]
            out = pkg.cached_attention(*new, *mine, ints(torch, pages), ints(torch, wrong), ints(torch, lens))
            assert bool(out[1:].isnan().all()) and bool(out[0].isfinite().all())
            untouched = np.ones(len(held), bool)
            untouched[pages[0]] = False
            for c, was in zip(mine, caches):
                assert torch.equal(c[torch.from_numpy(untouched).to("cuda")].nan_to_num(3.0),
                                   was[torch.from_numpy(untouched).to("cuda")].nan_to_num(3.0))
        bad = pages.copy()
        bad[0, 0], bad[1, 1], bad[2, 0], bad[3, 0] = -1, len(held), 2**31 - 1, -2**31
        check_attention(torch, pkg, new, newd, [c.clone() for c in caches], cachesd, bad, cached, None, "bf16")
        check_attention(torch, pkg, new, newd, [c.clone() for c in caches], cachesd, bad, cached, None, "bf16", left=2)


@pytest.mark.parametrize("dtype,B,L,Hq,Hkv,D,page,cached,left", [
    ("f16", 2, 1, 4, 1, 128, 64, [30011, 9000], None), ("bf16", 1, 1, 2, 2, 64, 16, [20000], 9000),
    ("f32", 1, 3, 2, 1, 64, 128, [12345], None), ("bf16", 3, 1, 1, 1, 96, 32, [7000, 0, 4096], None),
    ("bf16", 1, 100, 2, 1, 128, 16, [5000], None), ("f16", 2, 300, 4, 2, 64, 32, [1000, 1], 700)])
def test_attention_over_a_long_cache(torch, pkg, dtype, B, L, Hq, Hkv, D, page, cached, left):  # noqa: F811
    """Keys shared out among blocks, against float64 on the GPU; the sequences differ in length."""
    cached = np.array(cached)
    new, _, caches, _, pages, _ = attention_case(torch, B, L, Hq, Hkv, D, page, cached, None, dtype, 3)
    out = pkg.cached_attention(*new, *caches, ints(torch, pages), ints(torch, cached), left=left)
    tab = torch.from_numpy(pages).to("cuda")
    for b in range(B):
        S = int(cached[b]) + L
        j = torch.arange(S, device="cuda")
        k, v = (c[tab[b, j // page], :, j % page].double().transpose(0, 1).repeat_interleave(Hq // Hkv, 0) for c in caches)
        q, at = new[0][b].double().transpose(0, 1), torch.arange(L, device="cuda")[:, None] + int(cached[b])
        score = q @ k.transpose(1, 2) * D ** -0.5
        hidden = (j > at) | ((j < at - left) if left is not None else (j < 0))
        w = torch.softmax(score.masked_fill(hidden, -np.inf), -1)
        want, size = (w @ v).transpose(0, 1), (w @ v.abs()).transpose(0, 1)
        score_size = (q.abs() @ k.abs().transpose(1, 2)).amax(-1).transpose(0, 1)[..., None] * D ** -0.5
        want, size, score_size = (t.cpu().numpy() for t in (want, size, score_size))
        close(out[b], want, attention_tolerance(want, size, score_size, D, S, float(v.abs().max()), dtype), "out")


@pytest.mark.parametrize("dtype,L,Hkv", [(d, 60, 2) for d in DTYPES] + [("bf16", 300, 4)])
def test_attention_keys_of_many_rows_shared_by_few_blocks(torch, pkg, dtype, L, Hkv):  # noqa: F811
    """Two to eight blocks to a tile of rows; an utterance is empty, one has a single token, then one's length is bad."""
    cached, lens = np.array([600, 700, 0, 650, 3]), np.array([L, 0, 1, L - 21, L])
    new, newd, caches, cachesd, pages, _ = attention_case(torch, 5, L, 2 * Hkv, Hkv, 40, 32, cached, lens, dtype, L)
    out = check_attention(torch, pkg, new, newd, caches, cachesd, pages, cached, lens, dtype)
    for wrong in (-1, L + 1):
        lens[4] = wrong
        again = pkg.cached_attention(*new, *[c.clone() for c in caches], ints(torch, pages), ints(torch, cached), ints(torch, lens))
        assert torch.equal(again[:4], out[:4]) and bool(again[4].isnan().all())


def test_attention_offsets_past_32_bits(torch, pkg):  # noqa: F811
    """A cache of 6 GB: pages whose rows lie past 2^31 elements and 2^32 bytes."""
    D, page, Hkv = 128, 64, 2
    P = 190000
    caches = [torch.zeros((P, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pages = np.array([[P - 1, 0, P - 2], [P - 3, P // 2, 7]])
    g = torch.Generator(device="cuda").manual_seed(5)
    for c in caches:
        for p in pages.ravel():
            c[p] = torch.randn((Hkv, page, D), device="cuda", generator=g).bfloat16()
    small = [c[torch.from_numpy(pages.ravel()).to("cuda")].contiguous() for c in caches]
    q, k, v = (torch.randn((2, 5, h, D), device="cuda", generator=g).bfloat16() for h in (4, Hkv, Hkv))
    cached = ints(torch, [150, 60])
    out = pkg.cached_attention(q, k, v, *caches, ints(torch, pages), cached)
    want = pkg.cached_attention(q, k, v, *small, ints(torch, np.arange(6).reshape(2, 3)), cached)
    assert torch.equal(out, want)
    for c, s in zip(caches, small):
        assert torch.equal(c[torch.from_numpy(pages.ravel()).to("cuda")], s)


def test_attention_token_by_token(torch, pkg):  # noqa: F811
    """A sequence in one chunk, in chunks, and token by token over a shared first page: the same up to rounding, with
    the same cache at the end."""
    g = torch.Generator(device="cuda").manual_seed(6)
    N, D, page = 45, 64, 16
    q, k, v = (torch.randn((1, N, h, D), device="cuda", generator=g).half() for h in (4, 2, 2))
    pages = ints(torch, [[2, 0, 1]])
    results = []
    for cuts in ([N], [7, 1, 16, 21], [1] * N):
        caches = [torch.zeros((3, 2, page, D), dtype=torch.float16, device="cuda") for _ in range(2)]
        at, parts = 0, []
        cached = ints(torch, [0])
        for n in cuts:
            parts.append(pkg.cached_attention(q[:, at:at + n], k[:, at:at + n], v[:, at:at + n], *caches, pages, cached, left=30))
            cached += n
            at += n
        results.append((torch.cat(parts, 1), *caches))
    for out, kc, vc in results[1:]:
        assert torch.equal(kc, results[0][1]) and torch.equal(vc, results[0][2])
        # weights and results rounded to 2^-11, twice each
        assert bool(((out.float() - results[0][0].float()).abs() <= 6 * 2.0 ** -11 * 5).all())
    # two sequences that share their first pages and go on apart
    caches = [torch.zeros((5, 2, page, D), dtype=torch.float16, device="cuda") for _ in range(2)]
    pkg.cached_attention(q[:, :32], k[:, :32], v[:, :32], *caches, ints(torch, [[4, 2]]), ints(torch, [0]))
    two = [torch.cat([t[:, 32:], t[:, 32:].flip(1)]) for t in (q, k, v)]
    out = pkg.cached_attention(*two, *caches, ints(torch, [[4, 2, 0], [4, 2, 1]]), ints(torch, [32, 32]))
    for i in range(2):
        alone = [c.clone() for c in caches]
        assert torch.equal(out[i:i + 1], pkg.cached_attention(*[t[i:i + 1] for t in two], *alone, ints(torch, [[4, 2, i]]), ints(torch, [32])))


# ---------------------------------------------------------------- calls as programs make them

class Layer:
    """An encoder's layer in 8 bits: norm, queries, keys and values, positions, attention over the cache, its
    projection, norm, and a product of the width of the model."""

    def __init__(self, torch, pkg, B, L, H, D, dtype, seed):  # noqa: F811
        g = torch.Generator(device="cuda").manual_seed(seed)
        W = H * D
        self.pkg, self.B, self.L, self.H, self.D = pkg, B, L, H, D
        self.real = {n: torch.randn((m, W), device="cuda", generator=g) * W ** -0.5 for n, m in (("qkv", 3 * W), ("out", W), ("last", 29))}
        self.w8 = {n: pkg.quantize_rows(t) for n, t in self.real.items()}
        self.norm = [(1 + 0.2 * torch.randn((W,), device="cuda", generator=g)).to(dtype) for _ in range(2)]
        self.freq = pkg.rotary_frequencies(D)
        self.k_cache, self.v_cache = (torch.zeros((B * 4, H, 16, D), dtype=dtype, device="cuda") for _ in range(2))
        self.pages = torch.arange(B * 4, device="cuda", dtype=torch.int32).view(B, 4)
        self.cached = torch.zeros((B,), device="cuda", dtype=torch.int32)
        self.x = torch.randn((B, L, W), device="cuda", generator=g).to(dtype)
        self.before = torch.randn((B, L, W), device="cuda", generator=g).to(dtype)
        self.lens = torch.full((B,), L, device="cuda", dtype=torch.int32)

    def step(self):
        p = self.pkg
        rows, x = p.rms_norm8(self.x, self.norm[0], self.before, self.lens)
        q, k, v = p.linear8(rows, self.w8["qkv"], dtype=x.dtype).view(self.B, self.L, 3, self.H, self.D).unbind(2)
        q, k = (p.rotary(t, self.freq, self.cached, self.lens) for t in (q, k))
        out = p.cached_attention(q, k, v, self.k_cache, self.v_cache, self.pages, self.cached, self.lens, causal=False, left=20)
        rows, x = p.rms_norm8(p.linear8(out.flatten(2), self.w8["out"]), self.norm[1], x, self.lens)
        logits = p.linear8(rows, self.w8["last"], dtype=x.dtype)
        self.cached += self.lens
        return logits, x


def test_layer_against_float64(torch, pkg):  # noqa: F811
    """Three chunks through the layer in float32 with its weights' 8-bit values, against the same formulas in float64
    (activations there not in 8 bits, which are off by half a step of 1/127 of a row's largest value each)."""
    B, L, H, D = 2, 6, 2, 32
    layer = Layer(torch, pkg, B, L, H, D, torch.float32, 1)
    value = {n: (r.values.double() * r.scale.double()[:, None]).cpu().numpy() for n, r in layer.w8.items()}
    norm = [w.double().cpu().numpy() for w in layer.norm]
    freq, pages = layer.freq.cpu().numpy(), layer.pages.cpu().numpy()
    kc, vc = np.zeros((B * 4, H, 16, D)), np.zeros((B * 4, H, 16, D))
    for i in range(3):
        logits, x = layer.step()
        cached, lens = np.full(B, i * L), np.full(B, L)
        y, t = R.rms_norm(layer.x.double().cpu().numpy(), norm[0], layer.before.double().cpu().numpy(), lens)
        q, k, v = np.moveaxis((y @ value["qkv"].T).reshape(B, L, 3, H, D), 2, 0)
        q, k = (R.rotary(a, freq, cached, lens)[0] for a in (q, k))
        out, _, _, kc, vc = R.cached_attention(q, k, v, kc, vc, pages, cached, lens, causal=False, left=20)
        y, t = R.rms_norm(out.reshape(B, L, -1) @ value["out"].T, norm[1], t, lens)
        want = y @ value["last"].T
        # a product's 64 terms are each off by at most (max / 254) |w|: independent, their sum by about
        # sqrt(64) (max / 254) / sqrt(3) of one weight's size; two products and an attention lie behind each other
        assert np.sqrt(np.mean((x.double().cpu().numpy() - t) ** 2)) <= 0.02 * np.sqrt(np.mean(t ** 2))
        assert np.sqrt(np.mean((logits.double().cpu().numpy() - want) ** 2)) <= 0.03 * np.sqrt(np.mean(want ** 2))


def test_layer_captured_and_replayed(torch, pkg):  # noqa: F811
    """A step of the layer in a graph, replayed chunk after chunk, with eager work of another layer between."""
    for L in (1, 5):
        eager, kept, other = (Layer(torch, pkg, 3, L, 2, 64, torch.bfloat16, s) for s in (2, 2, 3))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            kept.step()
        torch.cuda.current_stream().wait_stream(side)
        kept.cached.zero_()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = kept.step()
        kept.cached.zero_()
        for _ in range(4):
            graph.replay()
            other.step()
            torch.cuda.synchronize()
            want = eager.step()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
            assert torch.equal(kept.k_cache, eager.k_cache) and torch.equal(kept.v_cache, eager.v_cache)
            x = torch.randn(eager.x.shape, device="cuda").to(eager.x.dtype)
            eager.x.copy_(x)
            kept.x.copy_(x)


def test_workspaces_of_two_graphs(torch, pkg):  # noqa: F811
    """Calls that take workspaces, captured side by side in two graphs and replayed in turn."""
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((4, 500, 96), device="cuda", generator=g, requires_grad=True)
    w = torch.randn((96,), device="cuda", generator=g, requires_grad=True)
    dy = torch.randn((4, 500, 96), device="cuda", generator=g)
    w8 = pkg.quantize_rows(torch.randn((70, 96), device="cuda", generator=g))
    freq = pkg.rotary_frequencies(32)
    heads = torch.randn((2, 30, 3, 32), device="cuda", generator=g, requires_grad=True)
    q, k, v = (torch.randn((1, 1, 2, 64), device="cuda", generator=g).half() for _ in range(3))
    caches = [torch.randn((300, 2, 64, 64), device="cuda", generator=g).half() for _ in range(2)]
    pages, cached = torch.arange(300, device="cuda", dtype=torch.int32)[None], ints(torch, [19000])

    def norm():
        y = pkg.rms_norm(x, w)
        return (y.detach(),) + torch.autograd.grad(y, (x, w), dy)

    def rotary():
        y = pkg.rotary(heads, freq)
        return (y.detach(),) + torch.autograd.grad(y, heads, torch.ones_like(y))

    def linear():
        return (pkg.linear8(x.detach(), w8),)

    def attention():
        return (pkg.cached_attention(q, k, v, *caches, pages, cached),)

    for fn in (norm, rotary, linear, attention):
        want = fn()
        torch.cuda.synchronize()
        want = [t.clone() for t in want]
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = fn()
            graphs.append((graph, out))
        for i in range(4):
            graph, out = graphs[i % 2]
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), fn.__name__
            again = fn()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(again, want))


@pytest.mark.parametrize("dtype", DTYPES)
def test_odd_addresses(torch, pkg, dtype):  # noqa: F811
    """Tensors that begin an element past an aligned address give the bits of aligned ones."""
    g = torch.Generator(device="cuda").manual_seed(10)

    def two(*shape):
        n = int(np.prod(shape))
        a = torch.randn(n + 1, device="cuda", generator=g).to(td(torch, dtype))[1:].view(shape)
        return a, a.clone()
    (x, x1), (r, r1), (w, w1), (dy, dy1) = two(3, 40, 136), two(3, 40, 136), two(136), two(3, 40, 136)
    for t in (x, x1, w, w1):
        t.requires_grad_(True)
    got, want = pkg.rms_norm(x, w, r), pkg.rms_norm(x1, w1, r1)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(got[0], (x, w), dy), torch.autograd.grad(want[0], (x1, w1), dy1)))
    x, x1, w, w1 = (t.detach() for t in (x, x1, w, w1))
    got, want = pkg.rms_norm8(x, w, r), pkg.rms_norm8(x1, w1, r1)
    assert torch.equal(got[0].values, want[0].values) and torch.equal(got[0].scale, want[0].scale) and torch.equal(got[1], want[1])
    assert torch.equal(pkg.quantize_rows(x).values, pkg.quantize_rows(x1).values)
    freq = pkg.rotary_frequencies(8)
    for inter in (False, True):
        assert torch.equal(pkg.rotary(x.view(3, 40, 8, 17), freq, interleaved=inter), pkg.rotary(x1.view(3, 40, 8, 17), freq, interleaved=inter))
    w8 = pkg.quantize_rows(torch.randn((70, 136), device="cuda", generator=g))
    (bias, bias1), (many, many1) = two(70), two(9000, 136)
    assert torch.equal(pkg.linear8(x, w8, bias), pkg.linear8(x1, w8, bias1))
    assert torch.equal(pkg.linear8(many, w8, bias), pkg.linear8(many1, w8, bias1))


def test_capture_without_a_workspace_is_refused(torch, pkg):  # noqa: F811
    """The C calls under a capture take no workspace of their own, and eagerly do."""
    enc = pkg.encoder
    lib = enc._library()
    x, w = torch.ones((40, 96), device="cuda"), torch.ones((96,), device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    wide = torch.ones((3000, 1040), device="cuda")
    w8 = pkg.quantize_rows(torch.ones((900, 1040), device="cuda"))
    y = torch.zeros((3000, 900), device="cuda")
    q, cache = torch.ones((1, 1, 2, 64), device="cuda"), torch.ones((100, 2, 64, 64), device="cuda")
    pages, cached, out = torch.arange(100, device="cuda", dtype=torch.int32), ints(torch, [6000]), torch.zeros((1, 1, 2, 64), device="cuda")
    ptr = lambda t: t.data_ptr()  # noqa: E731
    attention = enc.AttentionShape(1, 1, 2, 2, 64, 64, 100, 100, 1, -1, 0, *[128, 128, 64] * 3)

    def calls(stream):
        return (lib.rnnt_rms_norm_grad(ptr(x), None, enc.NormShape(1, 40, 96, 0), None, ptr(w), 1e-5, ptr(x), None, ptr(dx), ptr(dw), None, 0, stream),
                lib.rnnt_linear8_dynamic(ptr(wide), ptr(w8.values), ptr(w8.scale), enc.Linear8Shape(3000, 900, 1040, 0, 0, 1040), None, ptr(y), None, 0, stream),
                lib.rnnt_cached_attention(ptr(q), ptr(q), ptr(q), attention, None, ptr(cached), ptr(pages), ptr(cache), ptr(cache.clone()), 0.125, ptr(out), None, 0, stream))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        status = calls(torch.cuda.current_stream().cuda_stream)
        dx.zero_()
    assert status == (6, 6, 6)
    graph.replay()
    torch.cuda.synchronize()
    assert calls(torch.cuda.current_stream().cuda_stream) == (0, 0, 0)
    torch.cuda.synchronize()
    # rows of ones: dw = the sum of 40 rows of t r, y = 1040 (both scales 1 / 127), attention of ones
    r = (1 + 1e-5) ** -0.5
    assert bool(((dw - 40 * r).abs() <= 200 * ONE * 40).all()) and bool(((y - 1040).abs() <= 8 * ONE * 1040).all())
    assert bool(((out - 1).abs() <= 1e-4).all())


def test_two_streams_at_once(torch, pkg):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn((4, 3000, 640), device="cuda", generator=g).bfloat16()
    w8 = pkg.quantize_rows(torch.randn((320, 640), device="cuda", generator=g))
    q, k, v = (torch.randn((1, 2, 4, 64), device="cuda", generator=g).half() for _ in range(3))
    caches = [torch.randn((300, 4, 64, 64), device="cuda", generator=g).half() for _ in range(2)]
    pages, cached = torch.arange(300, device="cuda", dtype=torch.int32)[None], ints(torch, [19000])
    want = pkg.linear8(x, w8), pkg.cached_attention(q, k, v, *caches, pages, cached)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    mine = [caches, [c.clone() for c in caches]]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, c in zip(streams, mine):
            with torch.cuda.stream(s):
                got.append((pkg.linear8(x, w8), pkg.cached_attention(q, k, v, *c, pages, cached)))
    torch.cuda.synchronize()
    for out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_chain_of_training(torch, pkg):  # noqa: F811
    """Norm, positions and the transducer's own operators under one loss: gradients in float32 against differences in
    float64."""
    from oracle import network_ref as N
    from oracle import rnnt_ref
    B, T, U, H, D, V = 2, 5, 2, 2, 8, 6
    W = H * D
    rng = rng_of(9)
    names = ("x", "r", "norm", "pred", "wo")
    val = dict(zip(names, (rng.standard_normal(s).astype(np.float32).astype(np.float64) for s in (
        (B, T, W), (B, T, W), (W,), (B, U + 1, W), (W, V)))))
    leaf = {k: torch.from_numpy(v.astype(np.float32)).to("cuda").requires_grad_(True) for k, v in val.items()}
    labels, tl, ul = np.array([[1, 2], [3, 0]]), np.array([5, 4]), np.array([2, 1])
    start = np.array([3, 100000])
    freq = pkg.rotary_frequencies(D)
    y, t = pkg.rms_norm(leaf["x"], leaf["norm"], leaf["r"], ints(torch, tl))
    y = pkg.rotary(y.view(B, T, H, D), freq, ints(torch, start), ints(torch, tl)).view(B, T, W) + t
    logits = pkg.joint_hidden(y, leaf["pred"], ints(torch, tl), ints(torch, ul), "tanh") @ leaf["wo"]
    loss = pkg.rnnt_loss_autograd(logits, ints(torch, labels), ints(torch, tl), ints(torch, ul), reduction="sum")
    grads = torch.autograd.grad(loss, [leaf[k] for k in names])

    def reference(v):
        y, t = R.rms_norm(v["x"], v["norm"], v["r"], tl)
        y = R.rotary(y.reshape(B, T, H, D), freq.cpu().numpy(), start, tl)[0].reshape(B, T, W) + t
        h = N.joint_hidden(y, v["pred"], tl, ul, "tanh")
        return float(np.sum(rnnt_ref.rnnt_loss_grad(h @ v["wo"], labels, tl, ul, 0, "rnnt")[0]))
    want = reference(val)
    assert abs(float(loss.detach()) - want) <= 1e-5 * abs(want)
    for name, got in zip(names, grads):
        d = rng.standard_normal(val[name].shape)
        up, down = dict(val), dict(val)
        up[name], down[name] = val[name] + 1e-5 * d, val[name] - 1e-5 * d
        diff = (reference(up) - reference(down)) / 2e-5
        got = got.double().cpu().numpy()
        # float32 all along: a few 1e-6 of the terms, whose sizes add up to at most |g| |d|
        assert abs(np.sum(got * d) - diff) <= 1e-5 * np.sum(np.abs(got * d)) + 1e-6, name


def test_binding_refusals(torch, pkg):  # noqa: F811
    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    i = lambda *s: torch.ones(s, device="cuda", dtype=torch.int32)  # noqa: E731
    x, w, half = f(2, 3, 16), f(16), {"dtype": torch.float16}
    w8 = pkg.quantize_rows(f(5, 16))
    freq = pkg.rotary_frequencies(8)
    q, kv, cache = f(2, 3, 4, 8), f(2, 3, 2, 8), f(6, 2, 4, 8)

    def attend(**over):
        a = {"q": q, "k": kv, "v": kv, "k_cache": cache, "v_cache": cache.clone(), "pages": i(2, 3), "cached": i(2)}
        a.update(over)
        return pkg.cached_attention(**a)
    attend()
    narrow = torch.zeros((5, 40), dtype=torch.int8, device="cuda")
    for err, match, call in (
            (ValueError, "weight", lambda: pkg.rms_norm(x, f(8))), (TypeError, "weight", lambda: pkg.rms_norm(x, w.half())),
            (ValueError, "residual", lambda: pkg.rms_norm(x, w, f(2, 3, 8))), (ValueError, "eps", lambda: pkg.rms_norm(x, w, eps=-1.0)),
            (ValueError, "eps", lambda: pkg.rms_norm8(x, w, eps=float("nan"))), (ValueError, "contiguous", lambda: pkg.rms_norm(f(2, 16, 3).transpose(1, 2), w)),
            (ValueError, "lens", lambda: pkg.rms_norm(f(3, 16), w, None, i(3))), (ValueError, "lens", lambda: pkg.rms_norm(x, w, None, i(3))),
            (TypeError, "x must be float32", lambda: pkg.rms_norm(x.double(), w.double())),
            (RuntimeError, "no gradient", lambda: pkg.rms_norm8(f(2, 16, requires_grad=True), w)),
            (RuntimeError, "no gradient", lambda: pkg.quantize_rows(f(2, 16, requires_grad=True))),
            (RuntimeError, "no gradient", lambda: pkg.linear8(f(2, 16, requires_grad=True), w8)),
            (RuntimeError, "no gradient", lambda: attend(q=f(2, 3, 4, 8, requires_grad=True))),
            (TypeError, "weight must be Rows8", lambda: pkg.linear8(x, f(5, 16))), (ValueError, "x must be", lambda: pkg.linear8(f(2, 8), w8)),
            (TypeError, "bias", lambda: pkg.linear8(x, w8, f(5, **half))), (ValueError, "bias", lambda: pkg.linear8(x, w8, f(6))),
            (TypeError, "dtype", lambda: pkg.linear8(x, w8, dtype=torch.float16)),
            (ValueError, "one pitch", lambda: pkg.linear8(x, pkg.Rows8(narrow[:, :16], f(5)))),
            (ValueError, "one pitch", lambda: pkg.linear8(x, pkg.Rows8(torch.zeros((16, 16), dtype=torch.int8, device="cuda").t(), f(16)))),
            (ValueError, "pieces", lambda: pkg.linear8(f(2, 9), pkg.Rows8(torch.zeros((1, 9), dtype=torch.int8, device="cuda"), f(1)))),
            (TypeError, "int8", lambda: pkg.linear8(x, pkg.Rows8(f(5, 16), f(5)))), (ValueError, "scale", lambda: pkg.linear8(x, pkg.Rows8(w8.values, f(4)))),
            (ValueError, "B, L, H, D", lambda: pkg.rotary(x, freq)), (TypeError, "freq", lambda: pkg.rotary(q, freq.float())),
            (ValueError, "freq", lambda: pkg.rotary(q, pkg.rotary_frequencies(10))), (TypeError, "start", lambda: pkg.rotary(q, freq, f(2))),
            (ValueError, "channels", lambda: pkg.rotary(f(2, 3, 8, 4).transpose(2, 3), freq)), (ValueError, "lens", lambda: pkg.rotary(q, freq, None, i(3))),
            (ValueError, "even", lambda: pkg.rotary_frequencies(7)), (ValueError, "fast", lambda: pkg.rotary_frequencies(8, slow=4, fast=2)),
            (ValueError, "divisor", lambda: attend(k=f(2, 3, 3, 8), v=f(2, 3, 3, 8))), (ValueError, "divisor", lambda: attend(v=f(2, 3, 2, 4))),
            (TypeError, "k must be", lambda: attend(k=kv.half())), (ValueError, "k_cache", lambda: attend(k_cache=f(6, 1, 4, 8))),
            (ValueError, "v_cache", lambda: attend(v_cache=f(5, 2, 4, 8))), (TypeError, "pages", lambda: attend(pages=i(2, 3).long())),
            (ValueError, "pages", lambda: attend(pages=i(3, 3))), (ValueError, "cached", lambda: attend(cached=i(3))),
            (ValueError, "left", lambda: attend(left=-1)), (ValueError, "lens", lambda: attend(lens=i(1))),
            (pkg.RNNTError, "BAD_VARIANT", lambda: attend(scale=float("inf"))),
            (pkg.RNNTError, "UNSUPPORTED", lambda: attend(k_cache=f(6, 2, 3, 8), v_cache=f(6, 2, 3, 8))),
            (pkg.RNNTError, "UNSUPPORTED", lambda: pkg.cached_attention(f(1, 1, 1, 12), f(1, 1, 1, 12), f(1, 1, 1, 12), f(1, 1, 4, 12), f(1, 1, 4, 12), i(1, 1), i(1)))):
        with pytest.raises(err, match=match):
            call()
    leaf = f(2, 3, 16, requires_grad=True)
    y = pkg.rms_norm(leaf, w)
    (g,) = torch.autograd.grad(y, leaf, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), leaf)


# ---------------------------------------------------------------- values that lanes give one another

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [100, 256, 301, 512, 640, 767, 860, 1024])
def test_linear8_of_whole_numbers(torch, pkg, K, dtype):  # noqa: F811
    """Rows held in registers, of every width: with scales of 1 each result is a whole number, rounded once, and a row or a
    piece of one in another's place is seen.  The product in float64 is exact."""
    g = torch.Generator(device="cuda").manual_seed(K)
    M, N = 2100, 331
    x = torch.randint(-60, 61, (M, K), device="cuda", generator=g)
    x[torch.arange(M, device="cuda"), torch.randint(0, K, (M,), device="cuda", generator=g)] = 127  # the scale is 1
    w = pkg.quantize_rows(torch.cat([torch.randint(-126, 127, (N, K - 1), device="cuda", generator=g),
                                     torch.full((N, 1), 127, device="cuda")], 1).float())
    assert bool((w.scale == 1).all())
    want = (x.double() @ w.values.double().t()).to(td(torch, dtype))
    rows = pkg.quantize_rows(x.to(td(torch, dtype)))
    assert torch.equal(rows.values.long(), x)
    for _ in range(3):
        assert torch.equal(pkg.linear8(x.to(td(torch, dtype)), w), want)
        assert torch.equal(pkg.linear8(rows, w, dtype=td(torch, dtype)), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,L,cached", [(40, 5, 300), (64, 1, 777), (64, 16, 40), (128, 3, 2500), (200, 7, 130), (128, 150, 90), (64, 100, 900)])
def test_attention_of_one_key(torch, pkg, D, L, cached, dtype):  # noqa: F811
    """Every row's weights are 1 for one key, anywhere among those it sees, and 0 for the others: the row is that key's
    value, to the bit, and a value in another's place is seen."""
    g = torch.Generator(device="cuda").manual_seed(D + L)
    B, H, page = 2, 2, 16
    to, S = td(torch, dtype), cached + L
    k = torch.where(torch.rand((B, S, H, D), device="cuda", generator=g) < 0.5, -1.0, 1.0)
    v = torch.randint(-255, 256, (B, S, H, D), device="cuda", generator=g).float()
    to_key = torch.randint(0, S, (B, L, H), device="cuda", generator=g)
    pick = lambda t: torch.gather(t, 1, to_key[..., None].expand(-1, -1, -1, D))  # noqa: E731
    # keys of random signs agree in at most D - 8 more places than not, so the others' scores are 8 * 4 * 8 lower
    q = pick(k)
    agree = torch.einsum("blhd,bshd->blsh", q.cpu(), k.cpu()).to("cuda")
    agree.scatter_(2, to_key[:, :, None], -float(D))
    assert float(agree.max()) <= D - 8
    width = -(-S // page)
    pages = torch.randperm(B * width, device="cuda", generator=g).view(B, width)
    caches = []
    for t in (k, v):
        c = torch.zeros((B * width, H, page, D), dtype=to, device="cuda")
        at = torch.arange(cached, device="cuda")
        for b in range(B):
            c[pages[b, at // page], :, at % page] = t[b, :cached].to(to)
        caches.append(c)
    args = [t.to(to).contiguous() for t in (4 * q, k[:, cached:], v[:, cached:])]
    for _ in range(3):
        out = pkg.cached_attention(*args, *caches, pages.to(torch.int32), ints(torch, [cached] * B), causal=False, scale=8.0)
        assert torch.equal(out, pick(v).to(to))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("low,high", [(20, 26), (25.25, 26)])
@pytest.mark.parametrize("B,L,at", [(1, 1, 5), (600, 1, 5), (600, 1, 9000), (1, 100, 5), (260, 100, 5), (260, 100, 9000)])
def test_attention_of_many_small_weights(torch, pkg, B, L, at, low, high, dtype):  # noqa: F811
    """One key takes nearly all of the weight and has value 0; 9984 others, of weights down to 2^-26 of its own, make the
    result, in blocks that share them out and in one block.  Scores are exact, so a weight is off by the exponential's 2^-22, the
    exponent's 2^-18 (26 bits, 2^-23 each) and half a step of the values' type, or a whole one below 2^-25 of the largest, however
    many they are; besides there are float32's sums, of terms of one sign."""
    g = torch.Generator(device="cuda").manual_seed(B + L + at)
    N, D, page, to = 9984, 64, 64, td(torch, dtype)
    bits = torch.randint(int(low * 8), high * 8 + 1, (N,), device="cuda", generator=g).double() / 8
    bits[at] = 0
    v = (torch.rand((N, D), device="cuda", generator=g) * 0.5 + 0.5).to(to)
    v[at] = 0
    k = torch.zeros((N, D), device="cuda", dtype=to)
    k[:, 3] = -bits.to(to)
    # all utterances read the same pages; their new tokens, whose keys are too far down to count, go to pages of their own
    P, own = N // page, -(-L // page)
    pages = torch.randperm(P, device="cuda", generator=g)
    caches = [torch.zeros((P + B * own, 1, page, D), dtype=to, device="cuda") for _ in range(2)]
    for c, t in zip(caches, (k, v)):
        c[pages, 0] = t.view(P, page, D)
    table = torch.cat([pages.expand(B, P), P + torch.arange(B * own, device="cuda").view(B, own)], 1).to(torch.int32)
    q, new_k = torch.zeros((B, L, 2, D), device="cuda", dtype=to), torch.zeros((B, L, 1, D), device="cuda", dtype=to)
    q[..., 3], new_k[..., 3] = 1, -200
    out = pkg.cached_attention(q, new_k, torch.ones_like(new_k), *caches, table, ints(torch, [N] * B), scale=float(np.log(2.0)))
    w = torch.exp2(-bits)
    want = (w @ v.double()) / w.sum()
    weights = 0.0 if dtype == "f32" else 2 * HALF[dtype]
    tol = (HALF[dtype] + weights + 2.0 ** -18 + 2.0 ** -22 + (N + L) * ONE) * want + TINY[dtype]
    assert bool(((out.double() - want).abs() <= tol).all()), (float((out.double() / want).min()), float((out.double() / want).max()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L,G,cached", [(5, 1, 200), (100, 1, 200), (60, 2, 900)])
@pytest.mark.parametrize("scale", [1.0, 0.37, -0.61])
def test_attention_of_scores_of_billions(torch, pkg, L, G, cached, scale, dtype):  # noqa: F811
    """Scores whose last digit in float32 stands for hundreds of powers of two: every row has one key far above the others, so its
    weight is 1 and the row that key's value."""
    g = torch.Generator(device="cuda").manual_seed(L)
    D, page, to, S = 64, 16, td(torch, dtype), cached + L
    k = torch.where(torch.rand((1, S, 1, D), device="cuda", generator=g) < 0.5, -1.0, 1.0)
    v = torch.randint(-255, 256, (1, S, 1, D), device="cuda", generator=g).float()
    to_key = torch.randint(0, S, (1, L, G), device="cuda", generator=g)
    q = k[0, to_key[0], 0][None] * (1.0 if scale > 0 else -1.0)
    width = -(-S // page)
    pages = torch.arange(width, device="cuda", dtype=torch.int32)[None]
    caches = []
    for t in (5120 * k, v):
        c = torch.zeros((width * page, D), dtype=to, device="cuda")
        c[:cached] = t[0, :cached, 0].to(to)
        caches.append(c.view(width, 1, page, D))
    out = pkg.cached_attention((24576 * q).to(to), (5120 * k[:, cached:]).to(to), v[:, cached:].to(to), *caches, pages,
                               ints(torch, [cached]), causal=False, scale=scale)
    assert torch.equal(out, v[0, to_key[0], 0][None].to(to))


def test_rows_past_a_launch_along_x(torch, pkg):  # noqa: F811
    """4194307 rows of a block of 1024 lanes each are more threads than a launch takes along x."""
    n, D = (1 << 22) + 3, 8200
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GiB of GPU memory")
    g = torch.Generator(device="cuda").manual_seed(4)
    at = torch.tensor([0, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, n - 1], device="cuda")
    x = torch.ones((n, D), dtype=torch.bfloat16, device="cuda")
    x[at] = torch.randn((len(at), D), device="cuda", generator=g).bfloat16()
    w = torch.ones((D,), dtype=torch.bfloat16, device="cuda")
    for call in (pkg.quantize_rows, lambda t: pkg.rms_norm8(t, w)):
        rows, few, one = call(x), call(x[at]), call(x[1:2])
        assert torch.equal(rows.values[at], few.values) and torch.equal(rows.scale[at], few.scale)
        assert int((rows.scale != one.scale).sum()) == len(at)  # and every other row is one of ones
        del rows
    y = pkg.rms_norm(x, w)
    assert torch.equal(y[at], pkg.rms_norm(x[at], w)) and bool((y[2::999983] == y[1]).all())
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_gradient_of_bad_lengths(torch, pkg, interleaved, dtype):  # noqa: F811
    """A length outside its range: NaN in the utterance's results and 0 in its gradient, as the other operators have it."""
    x, xd = rounded(torch, rng_of(14).standard_normal((5, 3, 2, 21)), dtype)
    x.requires_grad_(True)
    freq, lens = pkg.rotary_frequencies(18), np.array([3, 4, -1, 2, -2**31])
    y = pkg.rotary(x, freq, None, ints(torch, lens), interleaved=interleaved)
    (dx,) = torch.autograd.grad(y, x, torch.ones_like(y))
    assert bool(y[[1, 2, 4]].isnan().all()) and bool(y[[0, 3]].isfinite().all())
    assert not bool(dx[[1, 2, 4]].any()) and not bool(dx[3, 2:].any())
    want, size = R.rotary(np.ones(xd.shape), freq.cpu().numpy(), None, np.array([3, 0, 0, 2, 0]), interleaved, -1.0)
    close(dx, want, HALF[dtype] * np.abs(want) + (2.0 ** -21 + 2 * ONE) * size + TINY[dtype] * (size > 0), "dx")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [5, 40, 1025])
def test_norm8_without_eps(torch, pkg, D, dtype):  # noqa: F811
    """With eps 0 a row of zeros is 0 / 0: NaN in the norm, and a scale of NaN in 8 bits."""
    x = torch.zeros((3, D), device="cuda", dtype=td(torch, dtype))
    x[1] = 2
    w = torch.ones((D,), device="cuda", dtype=td(torch, dtype))
    y, rows = pkg.rms_norm(x, w, eps=0.0), pkg.rms_norm8(x, w, eps=0.0)
    assert bool(y[0].isnan().all()) and bool((y[1] == 1).all())
    assert bool(rows.scale[[0, 2]].isnan().all()) and not bool(rows.values[[0, 2]].any())
    assert bool((rows.values[1] == 127).all()) and abs(float(rows.scale[1]) * 127 - 1) <= 4 * ONE


def test_product_in_8_bits_into_the_alignment(torch, pkg):  # noqa: F811
    """The joint's hidden layer through the 8-bit product into forced alignment: logits against float64, and the path of those
    logits against the oracle's."""
    from oracle import network_ref as N
    from oracle import rnnt_ref
    from oracle import viterbi as VB
    rng = rng_of(15)
    B, T, U, H, V = 3, 9, 4, 40, 21
    tl, ul = np.array([9, 6, 5]), np.array([4, 2, 0])
    labels = rng.integers(1, V, size=(B, U))
    enc, encd = rounded(torch, rng.standard_normal((B, T, H)), "bf16")
    pred, predd = rounded(torch, rng.standard_normal((B, U + 1, H)), "bf16")
    bias, biasd = rounded(torch, rng.standard_normal(V), "bf16")
    w8 = pkg.quantize_rows(torch.from_numpy(2 * rng.standard_normal((V, H))).to("cuda").float())
    hidden = pkg.joint_hidden(enc, pred, ints(torch, tl), ints(torch, ul), "tanh")
    logits = pkg.linear8(hidden, w8, bias)
    rows = pkg.quantize_rows(hidden)
    y, size = R.linear8(rows.values.reshape(-1, H).cpu().numpy(), rows.scale.reshape(-1).double().cpu().numpy(),
                        w8.values.cpu().numpy(), w8.scale.double().cpu().numpy(), biasd)
    close(logits.reshape(-1, V), y, HALF["bf16"] * np.abs(y) + 4 * ONE * size, "logits")
    # and the hidden layer itself, whose rows are 8 bits of it: half a step of each row's largest value, a bf16 rounding
    want = N.joint_hidden(encd, predd, tl, ul, "tanh")
    held = (rows.values.double() * rows.scale.double()[..., None]).cpu().numpy()
    most = np.abs(want).max(-1, keepdims=True)
    assert np.all(np.abs(held - want) <= (1 / 254 + 2 * HALF["bf16"]) * most + 1e-6)
    score, frames, span = pkg.viterbi_align(logits, ints(torch, labels), ints(torch, tl), ints(torch, ul))
    seen = logits.double().cpu().numpy()
    for b in range(B):
        z = seen[b, :tl[b], :ul[b] + 1]
        _, blank, label = rnnt_ref.lattice_weights(z, labels[b, :ul[b]], 0)
        best = VB.best_alignment(blank, label, "rnnt")
        assert abs(float(score[b]) - best["score"]) <= 1e-5 * max(1.0, abs(best["score"]))
        got = [int(f) for f in frames[b, :ul[b]]]
        assert bool((frames[b, ul[b]:] == -1).all())
        own = VB.alignment_score(blank, label, got, int(span[b, 0]), int(span[b, 1]), "rnnt")
        assert abs(own - best["score"]) <= 1e-5 * max(1.0, abs(best["score"]))


# tiles of 128 rows at every width of heads, and what a scale of 0 or below and a window do there; then tiles of 128 for 17 to 64
# rows, where utterances are many
WIDE = [  # B, L, Hq, Hkv, D, page, cached, lens, layout, options
    (2, 75, 1, 1, 72, 16, [21, 60], [75, 70], "dense", {}),
    (1, 71, 2, 1, 80, 8, [33], [69], "fused", {"left": 25}),
    (2, 150, 1, 1, 80, 16, [0, 40], [150, 1], "fused", {"causal": False, "left": 30}),
    (2, 70, 1, 1, 96, 16, [50, 3], [70, 67], "heads first", {"causal": False}),
    (1, 37, 4, 2, 96, 32, [20], [37], "fused", {}),
    (1, 130, 1, 1, 88, 16, [7], [129], "dense", {"left": 0}),
    (2, 75, 2, 2, 64, 16, [40, 0], [75, 33], "dense", {"scale": 0.0}),
    (2, 75, 2, 2, 64, 16, [40, 0], [75, 33], "fused", {"scale": -0.3}),
    (1, 90, 2, 1, 128, 16, [35], [87], "fused", {"scale": -0.3, "left": 40}),
    (1, 90, 1, 1, 32, 8, [35], None, "dense", {"scale": 0.0, "left": 17, "causal": False}),
    (1, 80, 1, 1, 24, 16, [300], [80], "dense", {"scale": 0.9, "left": 100})]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", WIDE, ids=lambda c: "-".join(map(str, c[:6])))
def test_attention_of_many_rows(torch, pkg, case, dtype):  # noqa: F811
    B, L, Hq, Hkv, D, page, cached, lens, layout, options = case
    cached, lens = np.array(cached), None if lens is None else np.array(lens)
    new, newd, caches, cachesd, pages, _ = attention_case(torch, B, L, Hq, Hkv, D, page, cached, lens, dtype, B + L + D, layout)
    check_attention(torch, pkg, new, newd, caches, cachesd, pages, cached, lens, dtype, **options)


def check_on_gpu(torch, pkg, dtype, B, L, Hq, Hkv, D, page, cached, lens=None, spare=2, **kw):  # noqa: F811
    """A call against float64 on the GPU; returns what it gave."""
    cached = np.array(cached)
    new, _, caches, _, pages, _ = attention_case(torch, B, L, Hq, Hkv, D, page, cached, lens, dtype, 3, spare=spare)
    out = pkg.cached_attention(*new, *caches, ints(torch, pages), ints(torch, cached), ints(torch, lens), **kw)
    tab, left, scale = torch.from_numpy(pages).to("cuda"), kw.get("left"), kw.get("scale", D ** -0.5)
    for b in range(B):
        n = L if lens is None else int(lens[b])
        assert not bool(out[b, n:].any())
        if not n:
            continue
        S = int(cached[b]) + n
        j = torch.arange(S, device="cuda")
        k, v = (c[tab[b, j // page], :, j % page].double().transpose(0, 1).repeat_interleave(Hq // Hkv, 0) for c in caches)
        q, at = new[0][b, :n].double().transpose(0, 1), torch.arange(n, device="cuda")[:, None] + int(cached[b])
        score = q @ k.transpose(1, 2).contiguous() * scale
        hidden = (j > at) if kw.get("causal", True) else (j < 0).expand(n, S)
        if left is not None:
            hidden = hidden | (j < at - left)
        w = torch.softmax(score.masked_fill(hidden, -np.inf), -1)
        want, size = (w @ v).transpose(0, 1), (w @ v.abs()).transpose(0, 1)
        score_size = (q.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1).transpose(0, 1)[..., None] * abs(scale)
        want, size, score_size = (t.cpu().numpy() for t in (want, size, score_size))
        close(out[b, :n], want, attention_tolerance(want, size, score_size, D, S, float(v.abs().max()), dtype), "out of %d" % b)
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L,D,options", [(20, 64, {}), (33, 40, {"causal": False}), (17, 96, {"left": 9}), (5, 128, {})])
def test_attention_of_many_streams(torch, pkg, L, D, options, dtype):  # noqa: F811
    """64 streams of 8 heads, some with no token: more tiles of sixteen rows than two to a CU, and waves that own no row."""
    rng = rng_of(L)
    lens, cached = rng.integers(0, L + 1, size=64), rng.integers(0, 60, size=64)
    lens[:3] = 0, L, 1
    check_on_gpu(torch, pkg, dtype, 64, L, 8, 8, D, 16, cached, lens, **options)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,L,Hq,Hkv,D,page,cached,lens,options", [
    # two to eight blocks to a tile, and more; sixteen rows to a tile, and 128; the chunk's tokens see one another
    (20, 3, 8, 4, 64, 16, [900] * 19 + [0], [3] * 18 + [0, 1], {"causal": False}),
    (1, 5, 2, 1, 64, 32, [3000], None, {"causal": False, "left": 1500}),
    (16, 100, 4, 4, 64, 16, [800] * 16, [100] * 15 + [37], {"causal": False}),
    (1, 130, 2, 2, 80, 16, [2500], [127], {"causal": False, "left": 2000}),
    # heads past 128 channels
    (1, 1, 2, 1, 256, 64, [4000], None, {}), (1, 9, 4, 2, 200, 32, [3001], [7], {"causal": False}),
    (20, 2, 4, 4, 256, 16, [1000] * 19 + [5], None, {}), (24, 3, 4, 4, 136, 16, [777] * 24, [3] * 23 + [0], {"left": 770}),
    # many splits of tables far wider than what they hold
    (1, 1, 4, 1, 64, 64, [80], None, {"spare": 900}), (3, 2, 2, 2, 128, 16, [0, 700, 31], [1, 2, 0], {"spare": 2000}),
    (20, 1, 8, 4, 64, 16, [30] * 20, None, {"spare": 100, "causal": False}), (2, 100, 2, 2, 64, 16, [30, 0], [100, 3], {"spare": 800}),
    (1, 2, 2, 1, 256, 16, [50], None, {"spare": 400})])
def test_attention_keys_shared_out(torch, pkg, B, L, Hq, Hkv, D, page, cached, lens, options, dtype):  # noqa: F811
    check_on_gpu(torch, pkg, dtype, B, L, Hq, Hkv, D, page, cached, None if lens is None else np.array(lens), **options)
