"""Float64 reference of the operators between an encoder and the transducer loss (label
embedding, gated recurrence, dropout, the joint's hidden layer), element by element from the
formulas, in numpy; it shares no code with the package.  Lengths outside their range give NaN
outputs and zero gradients for that utterance, rows behind a length are 0."""
import numpy as np


def _sigmoid(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


# ---------------------------------------------------------------- random numbers

M32 = 0xffffffff


def philox4x32(counter, key, rounds):
    """One block of Philox4x32 (Salmon et al., SC 2011) in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def numbers(block, seed, offset):
    """The eight 16-bit numbers of a block."""
    seed, offset = seed & (M32 << 32 | M32), offset & (M32 << 32 | M32)
    words = philox4x32([block & M32, block >> 32, offset & M32, offset >> 32], [seed & M32, seed >> 32], 7)
    return [words[i // 2] >> 16 * (i % 2) & 0xffff for i in range(8)]


def random16(n, seed, offset):
    """The 16-bit number of flat element n."""
    return numbers(n // 8, seed, offset)[n % 8]


def threshold(p):
    return min(int(np.rint(p * 65536.0)), 65535)


def keep_mask(shape, p, seed, offset, first=0):
    """Kept elements of a tensor whose flat numbering starts at `first`."""
    n, q = int(np.prod(shape)), threshold(p)
    blocks = {}
    out = np.empty(n, bool)
    for j in range(n):
        block, i = divmod(first + j, 8)
        if block not in blocks:
            blocks = {block: numbers(block, seed, offset)}
        out[j] = blocks[block][i] >= q
    return out.reshape(shape)


def dropout(x, p, seed, offset):
    return np.where(keep_mask(x.shape, p, seed, offset), x * (65536.0 / (65536.0 - threshold(p))), 0.0)


# ---------------------------------------------------------------- label embedding

def embedding_tokens(labels, lens, V, start):
    """Tokens of the output rows: -1 behind a length, -2 for a bad label or length."""
    B, N = labels.shape
    first = int(start is not None)
    out = np.full((B, N + first), -1, np.int64)
    for b in range(B):
        n = N if lens is None else int(lens[b])
        if not 0 <= n <= N:
            out[b] = -2
            continue
        if first:
            out[b, 0] = start
        for i in range(n):
            v = int(labels[b, i])
            out[b, first + i] = v if 0 <= v < V else -2
    return out


def label_embedding(labels, weight, lens=None, scale=1.0, start=None):
    tok = embedding_tokens(labels, lens, len(weight), start)
    out = np.zeros(tok.shape + (weight.shape[1],))
    out[tok == -2] = np.nan
    out[tok >= 0] = scale * weight[tok[tok >= 0]]
    return out


def label_embedding_grad(labels, V, dout, lens=None, scale=1.0, start=None):
    """(dweight, the sum of the absolute values of its terms)."""
    tok = embedding_tokens(labels, lens, V, start)
    dw = np.zeros((V, dout.shape[2]))
    size = np.zeros_like(dw)
    for b, i in np.argwhere(tok >= 0):
        dw[tok[b, i]] += dout[b, i]
        size[tok[b, i]] += np.abs(dout[b, i])
    return scale * dw, abs(scale) * size


# ---------------------------------------------------------------- gated recurrence

def gated_recurrence(x, z, h0=None, lens=None):
    B, L, D = x.shape
    h, last = np.zeros(x.shape), np.zeros((B, D))
    for b in range(B):
        n = L if lens is None else int(lens[b])
        s = np.zeros(D) if h0 is None else h0[b].astype(np.float64)
        if not 0 <= n <= L:
            h[b], last[b] = np.nan, np.nan
            continue
        for t in range(n):
            s = _sigmoid(z[b, t]) * s + _sigmoid(-z[b, t]) * x[b, t]
            h[b, t] = s
        last[b] = s
    return h, last


def gated_recurrence_grad(x, z, dh, dlast, h0=None, lens=None):
    """(dx, dz, dh0); dh, dlast None for zero."""
    B, L, D = x.shape
    dx, dz, dh0 = np.zeros(x.shape), np.zeros(x.shape), np.zeros((B, D))
    for b in range(B):
        n = L if lens is None else int(lens[b])
        if not 0 <= n <= L:
            continue
        s = np.zeros(D) if h0 is None else h0[b].astype(np.float64)
        before = []
        for t in range(n):
            before.append(s)
            s = _sigmoid(z[b, t]) * s + _sigmoid(-z[b, t]) * x[b, t]
        d = np.zeros(D) if dlast is None else dlast[b].astype(np.float64)
        for t in range(n - 1, -1, -1):
            a, g = _sigmoid(z[b, t]), _sigmoid(-z[b, t])
            if dh is not None:
                d = d + dh[b, t]
            dx[b, t] = g * d
            dz[b, t] = d * (before[t] - x[b, t]) * a * g
            d = a * d
        dh0[b] = d
    return dx, dz, dh0


# ---------------------------------------------------------------- the joint's hidden layer

def joint_hidden(enc, pred, logit_lens, label_lens, activation, p=0.0, seed=0, offset=0, dh=None):
    """h, or with dh (h, denc, dpred, the absolute sums of both)."""
    B, T, H = enc.shape
    U1 = pred.shape[1]
    h = np.zeros((B, T, U1, H))
    denc, dpred = np.zeros(enc.shape), np.zeros(pred.shape)
    senc, spred = np.zeros(enc.shape), np.zeros(pred.shape)
    scale = 65536.0 / (65536.0 - threshold(p))
    for b in range(B):
        tl, ul = int(logit_lens[b]), int(label_lens[b])
        if not (0 <= tl <= T and 0 <= ul < U1):
            h[b] = np.nan
            continue
        for t in range(tl):
            for u in range(ul + 1):
                s = enc[b, t].astype(np.float64) + pred[b, u]
                m = np.full(H, scale)
                if p > 0.0:
                    m = m * keep_mask((H,), p, seed, offset, ((b * T + t) * U1 + u) * H)
                if activation == "tanh":
                    val, slope = np.tanh(s), np.cosh(np.clip(s, -300, 300)) ** -2.0
                else:
                    val, slope = np.maximum(s, 0.0), (s > 0).astype(np.float64)
                h[b, t, u] = np.where(m > 0, m * val, 0.0)
                if dh is not None:
                    w = np.where(m * slope > 0, m * slope * dh[b, t, u], 0.0)
                    denc[b, t] += w
                    dpred[b, u] += w
                    senc[b, t] += np.abs(w)
                    spred[b, u] += np.abs(w)
    return h if dh is None else (h, denc, dpred, senc, spred)
