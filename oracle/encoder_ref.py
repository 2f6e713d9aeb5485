"""Float64 reference of the operators of an encoder's layers (root-mean-square norm, rows in 8
bits and their product, rotary positions, attention over a paged cache), element by element from
the formulas, in numpy; it shares no code with the package.  Rows behind a length are 0; lengths
outside their range give NaN outputs and zero gradients for that utterance."""
import numpy as np


def _lengths(lens, B, L):
    return [L if lens is None else int(lens[b]) for b in range(B)]


# ---------------------------------------------------------------- root-mean-square norm

def rms_norm(x, weight, residual=None, lens=None, eps=1e-5):
    """(y, t) over x (B, L, D)."""
    B, L, D = x.shape
    y, t = np.zeros(x.shape), np.zeros(x.shape)
    for b, n in enumerate(_lengths(lens, B, L)):
        if not 0 <= n <= L:
            y[b], t[b] = np.nan, np.nan
            continue
        for i in range(n):
            t[b, i] = x[b, i] if residual is None else x[b, i] + residual[b, i]
            y[b, i] = t[b, i] / np.sqrt(np.mean(t[b, i] ** 2) + eps) * weight
    return y, t


def rms_norm_grad(t, weight, dy, dsum=None, lens=None, eps=1e-5):
    """(dx, dweight, the sizes of the terms of both)."""
    B, L, D = t.shape
    dx, size, dw, dw_size = np.zeros(t.shape), np.zeros(t.shape), np.zeros(D), np.zeros(D)
    for b, n in enumerate(_lengths(lens, B, L)):
        if not 0 <= n <= L:
            continue
        for i in range(n):
            r = 1.0 / np.sqrt(np.mean(t[b, i] ** 2) + eps)
            unit, g = t[b, i] * r, dy[b, i] * weight
            dx[b, i] = r * (g - unit * np.mean(g * unit))
            size[b, i] = r * (np.abs(g) + np.abs(unit) * np.mean(np.abs(g * unit)))
            if dsum is not None:
                dx[b, i] += dsum[b, i]
                size[b, i] += np.abs(dsum[b, i])
            dw += dy[b, i] * unit
            dw_size += np.abs(dy[b, i] * unit)
    return dx, dw, size, dw_size


# ---------------------------------------------------------------- rows in 8 bits

def quantize_rows(x):
    """(the quotients 127 x / max, the scales) of rows (M, K); NaN scales where a row holds no number."""
    quotient, scale = np.zeros(x.shape), np.zeros(len(x))
    for m, row in enumerate(x):
        most = np.max(np.abs(row)) if np.all(np.isfinite(row)) else np.nan
        if np.isnan(most):
            scale[m] = np.nan
        elif most >= 2.0 ** -100:
            quotient[m], scale[m] = 127.0 * row / most, most / 127.0
    return quotient, scale


def linear8(q, q_scale, w, w_scale, bias=None):
    """(y, the size of what is added up last)."""
    total = q.astype(np.float64) @ w.astype(np.float64).T  # whole numbers below 2^53: exact
    y = total * q_scale[:, None] * w_scale[None]
    size = np.abs(y)
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    return y, size


# ---------------------------------------------------------------- rotary positions

def rotary(x, freq, start=None, lens=None, interleaved=False, sign=1.0):
    """(y, |a| + |b| of every turned channel, 0 of the others)."""
    B, L, H, D = x.shape
    R = 2 * len(freq)
    y, size = np.zeros(x.shape), np.zeros(x.shape)
    for b, n in enumerate(_lengths(lens, B, L)):
        if not 0 <= n <= L:
            y[b] = np.nan
            continue
        for t in range(n):
            y[b, t] = x[b, t]
            for i, f in enumerate(freq):
                one, two = (2 * i, 2 * i + 1) if interleaved else (i, R // 2 + i)
                angle = sign * ((0 if start is None else int(start[b])) + t) * f
                u, v = x[b, t, :, one], x[b, t, :, two]
                y[b, t, :, one] = u * np.cos(angle) - v * np.sin(angle)
                y[b, t, :, two] = u * np.sin(angle) + v * np.cos(angle)
                size[b, t, :, one] = size[b, t, :, two] = np.abs(u) + np.abs(v)
    return y, size


# ---------------------------------------------------------------- attention over a paged cache

def cached_attention(q, k, v, k_cache, v_cache, pages, cached, lens=None, scale=None, causal=True, left=None):
    """(out, sum of weights times |values|, the largest sum of |q k| scale of a row, k_cache, v_cache after the call)."""
    B, L, Hq, D = q.shape
    num_pages, Hkv, page, _ = k_cache.shape
    scale = D ** -0.5 if scale is None else scale
    out, size, score_size = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, L, Hq, 1))
    k_after, v_after = k_cache.copy(), v_cache.copy()

    def page_of(b, j):
        if j // page >= pages.shape[1]:
            return -1
        p = int(pages[b, j // page])
        return p if 0 <= p < num_pages else -1

    for b, n in enumerate(_lengths(lens, B, L)):
        c = int(cached[b])
        if not (0 <= n <= L and 0 <= c and c + n <= pages.shape[1] * page):
            out[b] = np.nan
            continue
        for t in range(n):
            p = page_of(b, c + t)
            if p >= 0:
                k_after[p, :, (c + t) % page], v_after[p, :, (c + t) % page] = k[b, t], v[b, t]
        for t in range(n):
            first = 0 if left is None else max(0, c + t - left)
            last = c + t if causal else c + n - 1
            for h in range(Hq):
                g = h // (Hq // Hkv)
                keys, values = np.full((last - first + 1, D), np.nan), np.full((last - first + 1, D), np.nan)
                for j in range(first, last + 1):
                    p = page_of(b, j)
                    if p >= 0:
                        keys[j - first] = k[b, j - c, g] if j >= c else k_cache[p, g, j % page]
                        values[j - first] = v[b, j - c, g] if j >= c else v_cache[p, g, j % page]
                with np.errstate(invalid="ignore", over="ignore"):
                    score = scale * (keys @ q[b, t, h])
                    w = np.exp(score - np.max(score))
                    w = w / np.sum(w)
                    out[b, t, h] = w @ values
                    size[b, t, h] = w @ np.abs(values)
                    score_size[b, t, h] = np.max(np.abs(scale) * (np.abs(keys) @ np.abs(q[b, t, h])))
    return out, size, score_size, k_after, v_after
