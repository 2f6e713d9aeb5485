"""Timed operators of a streaming encoder in serving and of its layers in training: the
root-mean-square norm (with the residual's addition, and in 8 bits with a scale a row), the
product in 8-bit integers, rotary positions, and the attention of a chunk of new tokens over a
paged cache.

A case is a dict of plain values; listed() names the fixed ones and draw() makes more from
the ranges they stand for.  prepare() builds what the caller's program holds before the
call, run() is one call (forward, or forward and backward), in the operators' plain form or,
with `own` set, through the package; exact() gives the same results in float64.

Keys of a case
  op        "norm", "linear", "rotary", "attend"
  mode      "infer" (forward alone), "train" (forward, then the gradients), "infer8" (the norm's
            output in 8 bits)
  dtype     "f32", "bf16", "f16": activations, weights and their gradients
  lengths   "full", or "variable" (new tokens 0.5-1 of the padded length, cached ones 0.3-1),
            drawn from len_seed, so a case has the same lengths for every input seed
  norm        B, L, D, residual
  linear      M rows, K, N, bias: rows in `dtype`, weights in 8 bits
  rotary      B, L, H, D, R rotated channels of a head, interleaved, far (positions start below it)
  attend      B, L new tokens, Hq, Hkv, D, page, cached, left (-1: all), causal
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
EXACT_MULTS = 1 << 41  # above this many multiplications the float64 result takes too long


def _norm(name, mode, B, L, D, dtype, residual, lengths="variable", len_seed=0):
    return {"name": name, "op": "norm", "mode": mode, "B": B, "L": L, "D": D, "dtype": dtype, "residual": residual,
            "lengths": lengths, "len_seed": len_seed}


def _linear(name, M, K, N, dtype, bias):
    return {"name": name, "op": "linear", "mode": "infer", "M": M, "K": K, "N": N, "dtype": dtype, "bias": bias}


def _rotary(name, mode, B, L, H, D, R, dtype, interleaved, far, lengths="variable", len_seed=0):
    return {"name": name, "op": "rotary", "mode": mode, "B": B, "L": L, "H": H, "D": D, "R": R, "dtype": dtype,
            "interleaved": interleaved, "far": far, "lengths": lengths, "len_seed": len_seed}


def _attend(name, B, L, Hq, Hkv, D, page, cached, dtype, causal, left=-1, lengths="variable", len_seed=0):
    return {"name": name, "op": "attend", "mode": "infer", "B": B, "L": L, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "cached": cached, "dtype": dtype, "causal": causal, "left": left, "lengths": lengths, "len_seed": len_seed}


def listed():
    return [
        # one step of a streaming decoder in 8 bits: the last token of each of 16 utterances
        _norm("norm_step", "infer8", 16, 1, 640, "f16", True, lengths="full"),
        # a batch of recordings recognised offline in 8 bits
        _norm("norm_batch", "infer8", 32, 1500, 640, "bf16", True, len_seed=1),
        # a training step over the encoder activations of a large batch
        _norm("norm_large", "train", 64, 1000, 1024, "bf16", True, len_seed=2),
        # one step of a streaming decoder: the projection to the word pieces
        _linear("linear_step", 16, 640, 1025, "f16", True),
        # a chunk of 16 frames of each of 64 live streams through a feed-forward layer
        _linear("linear_chunk", 1024, 512, 2048, "bf16", True),
        # the logits of a batch for forced alignment: every frame against every unit
        _linear("linear_joint", 32 * 250 * 81, 640, 1025, "bf16", False),
        # one step of a streaming decoder: queries and keys of one token, far into a recording
        _rotary("rotary_step", "infer", 16, 1, 16, 64, 64, "f16", False, 200003, lengths="full"),
        # a training step over the queries and keys of a batch of utterances
        _rotary("rotary_bpe", "train", 32, 250, 16, 64, 32, "bf16", True, 1, len_seed=3),
        # one step of a label decoder: one token of each of 16 utterances against its transcript so far
        _attend("attend_step", 16, 1, 8, 8, 64, 16, 80, "f32", True, len_seed=4),
        # a chunk of 16 frames of each of 64 live streams, 256 frames of left context
        _attend("attend_chunk", 64, 16, 8, 8, 64, 16, 1500, "bf16", False, left=256, len_seed=5),
        # one token against a whole recording, a few of them at once
        _attend("attend_long", 3, 1, 16, 2, 128, 64, 60013, "f16", True, lengths="full"),
        # long segments appended to recordings that are under way
        _attend("attend_batch", 8, 1500, 16, 4, 128, 32, 1000, "bf16", True, len_seed=6),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, sizes spread over the listed cases' ranges."""
    op = rng.choice(["norm", "linear", "rotary", "attend", "attend"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    lengths = rng.choice(["variable", "variable", "full"])
    len_seed = rng.randrange(1 << 20)
    width = rng.choice([_log_int(rng, 33, 2048), 64 * rng.randint(2, 32)])
    while True:
        B, L = _log_int(rng, 1, 64), _log_int(rng, 1, 1500)
        if op == "norm":
            mode = rng.choice(["infer", "infer8", "train", "train"])
            if mode == "infer8" and dtype == "f32":
                dtype = "bf16"  # 8 bits serve models of 16
            if B * L * width * BYTES[dtype] <= 64 * 1000 * 1024 * 2:
                return _norm("", mode, B, L, width, dtype, rng.random() < 0.7, lengths, len_seed)
        elif op == "linear":
            M, N = _log_int(rng, 1, 32 * 250 * 81), rng.choice([_log_int(rng, 29, 4096), 64 * rng.randint(2, 32)])
            if M * width * N <= 32 * 250 * 81 * 640 * 1025 and M * (width + N) * BYTES[dtype] <= 32 * 250 * 81 * 1665 * 2:
                return _linear("", M, width, N, dtype, rng.random() < 0.5)
        elif op == "rotary":
            D, H = 8 * rng.randint(4, 16), rng.randint(1, 24)
            R = rng.choice([D, D, 2 * rng.randint(1, D // 2)])
            if B * L * H * D * BYTES[dtype] <= 64 * 1000 * 1024 * 2:
                return _rotary("", rng.choice(["infer", "train"]), B, L, H, D, R, dtype, rng.random() < 0.5,
                               _log_int(rng, 1, 400000), lengths, len_seed)
        else:
            L = rng.choice([1, L])  # half of the calls are single tokens
            D, Hkv, G = rng.choice([32, 64, 64, 80, 96, 128]), rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 8])
            cached = _log_int(rng, 1, 60014) - 1
            left = rng.choice([-1, -1, _log_int(rng, 1, 1000)])
            rows = B * (cached + L) * Hkv * D * BYTES[dtype]
            pairs = B * L * (cached + L) * Hkv * G * (4 if dtype == "f32" else 1)
            if rows <= 3 * 60014 * 2 * 128 * 2 and pairs <= 8 * 1500 * 2500 * 16:
                return _attend("", B, L, Hkv * G, Hkv, D, rng.choice([8, 16, 32, 64, 128]), cached, dtype,
                               rng.random() < 0.6, left, lengths, len_seed)


# ---------------------------------------------------------------- inputs

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _lengths(case, padded, least, salt, longest):
    """(B,) lengths in [least * padded, padded]; with `longest` utterance 0 has the padded length."""
    B = case["B"]
    if case["lengths"] == "full":
        return np.full(B, padded, np.int32)
    rng = np.random.Generator(np.random.PCG64([salt, case["len_seed"], B, padded]))
    out = rng.integers(math.ceil(least * padded), padded, size=B, endpoint=True)
    if longest:
        out[0] = padded
    return out.astype(np.int32)


def _case_lengths(case):
    """The new tokens of every utterance, and for the attention the cached ones before them."""
    if case["op"] == "linear":
        return ()
    new = _lengths(case, case["L"], 0.5, 31, True)
    if case["op"] != "attend":
        return (new,)
    return new, _lengths(case, case["cached"], 0.3, 32, False)


def _inputs(case, seed):
    """The case's tensors for one seed."""
    dev, dtype = _device(), DTYPES[case["dtype"]]
    rng = np.random.Generator(np.random.PCG64([13, seed]))
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(rng.integers(1 << 40)))

    def normal(shape, sigma=1.0, mean=0.0, to=dtype):
        return torch.empty(shape, dtype=torch.float32, device=dev).normal_(mean, sigma, generator=gen).to(to)

    s = {}
    lens = [torch.from_numpy(x).to(dev) for x in _case_lengths(case)]
    train = case["mode"] == "train"
    if lens:
        # a program whose chunks are always whole passes no lengths
        s["lens"] = None if case["lengths"] == "full" else lens[0]
    if case["op"] == "norm":
        shape = (case["B"], case["L"], case["D"])
        s["x"], s["weight"] = normal(shape), normal((case["D"],), 0.2, 1.0)
        s["residual"] = normal(shape, 2.0) if case["residual"] else None
        if train:
            s["dy"] = normal(shape, 0.02)
            s["dsum"] = normal(shape, 0.02) if case["residual"] else None
    elif case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        # rows of different sizes, as the hidden layer of a joint or a feed-forward layer has them
        s["x"] = torch.empty((M, K), dtype=dtype, device=dev)
        for at in range(0, M, 1 << 17):  # drawn in float32, then rounded
            n = min(1 << 17, M - at)
            s["x"][at:at + n] = normal((n, K), to=torch.float32) * normal((n, 1), 0.5, to=torch.float32).exp_()
        # the weights' rows begin at multiples of 16 bytes
        s["w8"] = torch.zeros((N, -(-K // 16) * 16), dtype=torch.int8, device=dev)[:, :K]
        s["w8"].copy_(torch.randint(-127, 128, (N, K), generator=gen, device=dev))
        s["wscale"] = torch.empty((N,), dtype=torch.float32, device=dev).uniform_(0.5, 1.5, generator=gen) / (73.0 * math.sqrt(K))
        s["bias"] = normal((N,), 0.5) if case["bias"] else None
    elif case["op"] == "rotary":
        shape = (case["B"], case["L"], case["H"], case["D"])
        s["x"] = normal(shape)
        s["freq"] = 10000.0 ** (-torch.arange(0, case["R"], 2, dtype=torch.float64, device=dev) / case["R"])
        s["start"] = torch.from_numpy(rng.integers(0, case["far"], size=case["B"]).astype(np.int32)).to(dev)
        if train:
            s["dy"] = normal(shape, 0.02)
    else:
        B, L, Hkv, D, page = case["B"], case["L"], case["Hkv"], case["D"], case["page"]
        s["q"], s["k"], s["v"] = normal((B, L, case["Hq"], D)), normal((B, L, Hkv, D)), normal((B, L, Hkv, D))
        width = -(-(case["cached"] + L) // page)
        P = B * width + 3  # a few free pages too
        s["k_cache"], s["v_cache"] = normal((P, Hkv, page, D)), normal((P, Hkv, page, D))
        s["pages"] = torch.from_numpy(rng.permutation(P)[:B * width].reshape(B, width).astype(np.int32)).to(dev)
        s["cached"] = lens[1]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["mode"] == "train":
        for k in ("x", "weight", "residual"):
            if s.get(k) is not None:
                s[k].requires_grad_(True)
    return s


def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    with torch.no_grad():
        return {"norm": _plain_norm, "linear": _plain_linear, "rotary": _plain_rotary, "attend": _plain_attend}[case["op"]](case, s)


# ---------------------------------------------------------------- the package's operators

def _run_own(case, s):
    import paper_2303_10384_amd as rnnt
    train = case["mode"] == "train"
    op = case["op"]
    if op == "norm":
        if case["mode"] == "infer8":
            got = rnnt.rms_norm8(s["x"], s["weight"], s["residual"], s["lens"], eps=EPS)
            rows, total = got if case["residual"] else (got, None)
            # the values that the 8 bits stand for
            y = torch.mul(rows.values, rows.scale[..., None], out=torch.empty_like(s["x"]))
            return (y, total) if case["residual"] else y
        got = rnnt.rms_norm(s["x"], s["weight"], s["residual"], s["lens"], eps=EPS)
        if not train:
            return got
        if not case["residual"]:
            return (got.detach(),) + torch.autograd.grad(got, (s["x"], s["weight"]), s["dy"])
        return tuple(t.detach() for t in got) + torch.autograd.grad(got, (s["x"], s["weight"], s["residual"]),
                                                                    (s["dy"], s["dsum"]))
    if op == "linear":
        return rnnt.linear8(s["x"], rnnt.Rows8(s["w8"], s["wscale"]), s["bias"])
    if op == "rotary":
        y = rnnt.rotary(s["x"], s["freq"], s["start"], s["lens"], interleaved=case["interleaved"])
        return (y.detach(),) + torch.autograd.grad(y, s["x"], s["dy"]) if train else y
    out = rnnt.cached_attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["pages"], s["cached"], s["lens"],
                                causal=case["causal"], left=None if case["left"] < 0 else case["left"])
    return out, s["k_cache"], s["v_cache"]


# ---------------------------------------------------------------- plain forms

def _valid(case, s, device):
    """(B, L) which of the new tokens there are."""
    at = torch.arange(case["L"], device=device)[None]
    return (at < s["lens"].long()[:, None]) if s["lens"] is not None else (at < case["L"]).expand(case["B"], case["L"])


def _plain_norm(case, s):
    x, w = s["x"], s["weight"].float()
    valid = _valid(case, s, x.device)[..., None]
    zero = torch.zeros((), device=x.device)
    total = x.float() + s["residual"].float() if case["residual"] else x.float()
    total = torch.where(valid, total, zero)
    r = torch.rsqrt((total * total).mean(-1, keepdim=True) + EPS)
    y = total * r * w
    if case["mode"] == "infer8":
        most = y.abs().amax(-1, keepdim=True)
        y = torch.round(y * 127.0 / torch.where(most > 0, most, zero + 1.0)) * (most / 127.0)
    y, kept = y.to(x.dtype), total.to(x.dtype)
    if case["mode"] != "train":
        return (y, kept) if case["residual"] else y
    dy = torch.where(valid, s["dy"].float(), zero)
    unit = total * r
    g = dy * w
    dx = r * (g - unit * (g * unit).mean(-1, keepdim=True))
    dw = (dy * unit).sum((0, 1)).to(x.dtype)
    if not case["residual"]:
        return y, dx.to(x.dtype), dw
    dx = (dx + torch.where(valid, s["dsum"].float(), zero)).to(x.dtype)
    return y, kept, dx, dw, dx.clone()


def _plain_linear(case, s):
    x = s["x"].float()
    most = x.abs().amax(-1, keepdim=True)
    q = torch.round(x * 127.0 / torch.where(most > 0, most, torch.ones_like(most)))
    y = (q @ s["w8"].float().t()) * (most / 127.0) * s["wscale"]
    if case["bias"]:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


def _turned(x, case, cos, sin):
    """The pairs of the first R channels turned; float32."""
    R = case["R"]
    x = x.float()
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_rotary(case, s):
    x = s["x"]
    at = s["start"].double()[:, None] + torch.arange(case["L"], device=x.device, dtype=torch.float64)
    angle = at[..., None] * s["freq"]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    valid = _valid(case, s, x.device)[:, :, None, None]
    zero = torch.zeros((), device=x.device)
    y = torch.where(valid, _turned(x, case, cos, sin), zero).to(x.dtype)
    if case["mode"] == "infer":
        return y
    return y, torch.where(valid, _turned(s["dy"], case, cos, -sin), zero).to(x.dtype)


def _plain_attend(case, s):
    B, L, Hq, Hkv, D, page = (case[k] for k in ("B", "L", "Hq", "Hkv", "D", "page"))
    q, dev = s["q"], s["q"].device
    valid, cached, pages = _valid(case, s, dev), s["cached"].long(), s["pages"].long()
    at = cached[:, None] + torch.arange(L, device=dev)  # (B, L) positions of the new tokens
    row = torch.gather(pages, 1, torch.clamp_max(at // page, pages.shape[1] - 1))
    for cache, new in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])):
        cache[row[valid], :, (at % page)[valid]] = new[valid]
    S = pages.shape[1] * page
    k, v = (c[pages].transpose(1, 2).reshape(B, Hkv, S, D).float() for c in (s["k_cache"], s["v_cache"]))
    x = q.float().view(B, L, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * L, D)
    score = (x @ k.transpose(2, 3)).view(B, Hq, L, S) * (D ** -0.5)
    key = torch.arange(S, device=dev)
    ends = cached + valid.sum(1)
    seen = (key <= at[..., None]) if case["causal"] else (key < ends[:, None, None]).expand(B, L, S)
    if case["left"] >= 0:
        seen = seen & (key >= at[..., None] - case["left"])
    score = score.masked_fill_(~(seen & valid[..., None])[:, None], -math.inf)
    score = torch.exp_(score.sub_(score.amax(-1, keepdim=True)))
    out = score.view(B, Hkv, Hq // Hkv * L, S) @ v
    out = out.view(B, Hq, L, D) / score.sum(-1, keepdim=True)
    out = torch.where(valid[:, None, :, None], out, torch.zeros((), device=dev))
    return out.transpose(1, 2).contiguous().to(q.dtype), s["k_cache"], s["v_cache"]


# ---------------------------------------------------------------- what a pass cannot do without

def _seen(case):
    """(cached rows that some query of a sequence sees, pairs of query and key) summed over the batch."""
    new, cached = (x.astype(np.int64) for x in _case_lengths(case))
    rows = pairs = 0
    for n, c in zip(new.tolist(), cached.tolist()):
        at = c + np.arange(n, dtype=np.int64)
        first = np.maximum(0, at - case["left"]) if case["left"] >= 0 else np.zeros_like(at)
        last = at if case["causal"] else np.full_like(at, c + n - 1)
        pairs += int((last - first + 1).sum())
        rows += max(0, c - int(first[0]))
    return rows, pairs


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K * e + N * K + 4 * N + (N * e if case["bias"] else 0) + M * N * e, "flops": 2 * M * K * N}
    new = int(_case_lengths(case)[0].astype(np.int64).sum())
    padded = case["B"] * case["L"]
    if case["op"] == "norm":
        D, two = case["D"], int(case["residual"])
        n = new * D * e * (1 + two) + D * e + padded * D * e * two
        n += padded * (D + 4) if case["mode"] == "infer8" else padded * D * e
        if case["mode"] == "train":
            n += new * D * e * (2 + two) + padded * D * e + 2 * D * e
        return {"bytes": n, "flops": new * D * (14 if case["mode"] == "train" else 6)}
    if case["op"] == "rotary":
        row, times = case["H"] * case["D"] * e, 2 if case["mode"] == "train" else 1
        return {"bytes": times * (new + padded) * row + 4 * case["R"], "flops": times * 3 * new * case["H"] * case["R"]}
    rows, pairs = _seen(case)
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    n = 2 * rows * Hkv * D * e + 4 * new * Hkv * D * e + (new + padded) * Hq * D * e + 4 * rows // case["page"]
    return {"bytes": n, "flops": 4 * pairs * Hq * D}


# ---------------------------------------------------------------- the same in float64

def _exact_norm(case, s):
    B, L, D = s["x"].shape
    w, dev = s["weight"].detach().double(), s["x"].device
    y, kept, dx = (torch.zeros((B, L, D), dtype=torch.float64, device=dev) for _ in range(3))
    dw = torch.zeros((D,), dtype=torch.float64, device=dev)
    for b in range(B):
        n = L if s["lens"] is None else int(s["lens"][b])
        t = s["x"][b, :n].detach().double()
        if case["residual"]:
            t = t + s["residual"][b, :n].detach().double()
        size = torch.sqrt((t ** 2).sum(-1, keepdim=True) / D + EPS)
        out = w * t / size
        if case["mode"] == "infer8":
            most = out.abs().max(-1, keepdim=True).values
            out = torch.round(127 * out / torch.where(most > 0, most, 1.0)) * most / 127
        y[b, :n], kept[b, :n] = out, t
        if case["mode"] == "train":
            dy = s["dy"][b, :n].double()
            dx[b, :n] = w * dy / size - t * (w * dy * t).sum(-1, keepdim=True) / (D * size ** 3)
            if case["residual"]:
                dx[b, :n] += s["dsum"][b, :n].double()
            dw += (dy * t / size).sum(0)
    if case["mode"] != "train":
        return (y, kept) if case["residual"] else y
    return (y, kept, dx, dw, dx) if case["residual"] else (y, dx, dw)


def _exact_linear(case, s):
    w = s["w8"].double() * s["wscale"].double()[:, None]
    out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=w.device)
    for at in range(0, case["M"], 1 << 16):
        x = s["x"][at:at + (1 << 16)].double()
        most = x.abs().max(1, keepdim=True).values
        out[at:at + (1 << 16)] = (torch.round(127 * x / torch.where(most > 0, most, 1.0)) * most / 127) @ w.t()
    return out + s["bias"].double() if case["bias"] else out


def _exact_rotary(case, s):
    half = case["R"] // 2
    got = []
    for t, sign in ((s["x"], 1.0),) + (((s["dy"], -1.0),) if case["mode"] == "train" else ()):
        y = t.detach().double()
        for b in range(case["B"]):
            n = case["L"] if s["lens"] is None else int(s["lens"][b])
            y[b, n:] = 0
            at = int(s["start"][b]) + torch.arange(n, dtype=torch.float64, device=y.device)
            turn = torch.exp(1j * sign * at[:, None] * s["freq"])[:, None]
            z = y[b, :n, :, :case["R"]]
            if case["interleaved"]:
                y[b, :n, :, :case["R"]] = torch.view_as_real(torch.view_as_complex(z.unflatten(-1, (half, 2)).contiguous()) * turn).flatten(-2)
            else:
                c = torch.complex(z[..., :half], z[..., half:]) * turn
                y[b, :n, :, :half], y[b, :n, :, half:case["R"]] = c.real, c.imag
        got.append(y)
    return tuple(got) if len(got) > 1 else got[0]


def _exact_attend(case, s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    caches = [s["k_cache"].double(), s["v_cache"].double()]
    group, page = case["Hq"] // case["Hkv"], case["page"]
    for b in range(case["B"]):
        n = case["L"] if s["lens"] is None else int(s["lens"][b])
        c = int(s["cached"][b])
        key = torch.arange(c + n, device=out.device)
        where = (s["pages"][b].long()[key // page], key % page)
        both = []
        for cache, new in zip(caches, (s["k"], s["v"])):
            cache[where[0][c:], :, where[1][c:]] = new[b, :n].double()
            both.append(cache[where[0], :, where[1]])
        at = c + torch.arange(n, device=out.device)[:, None]
        hidden = key > at if case["causal"] else torch.zeros((n, c + n), dtype=torch.bool, device=out.device)
        if case["left"] >= 0:
            hidden = hidden | (key < at - case["left"])
        for h in range(case["Hq"]):
            score = s["q"][b, :n, h].double() @ both[0][:, h // group].t() / math.sqrt(case["D"])
            out[b, :n, h] = torch.softmax(score.masked_fill(hidden, -math.inf), 1) @ both[1][:, h // group]
    return out, caches[0], caches[1]


def exact(case, seed):
    w = work(case)
    if w["flops"] > EXACT_MULTS:
        return None
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "rotary": _exact_rotary, "attend": _exact_attend}[case["op"]](case, s)
