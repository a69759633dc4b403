"""The operators over plain arrays in 64 bits (numpy), from their definitions in include/pb.h, and bounds of the error of
32-bit kernels.  EPS is half a unit in the last place relative to a value: the error of one rounding."""
import numpy as np

EPS = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}      # the rounding to an output type
TINY = 2.0 ** -126                                         # results below the smallest normal number may be lost
BLOCK = 128


def scaled(x, scale):
    """scale * logit, which is a 32-bit product: infinite beyond their range."""
    xs = x * scale
    return np.where(np.abs(xs) > np.finfo(np.float32).max, np.copysign(np.inf, xs), xs)


def f64(t):
    return t.detach().double().cpu().numpy()


def padded(n):
    return -(-n // BLOCK) * BLOCK


# ------------------------------------------------------------------------------------------------------- 8-bit moments
def _mix(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def dither(n, seed, step, start=0):
    """Of the elements from place `start` on."""
    with np.errstate(over="ignore"):
        key = _mix(np.array([seed], np.uint64) ^ _mix(np.array([step], np.uint64)))
        i = np.arange(n, dtype=np.uint64) + np.uint64(start)
        z = _mix((i >> np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15) + key) >> (np.uint64(32) * (i & np.uint64(1)))
    return ((z & np.uint64(0xFFFF)).astype(np.int64) << 4 | 8), ((z >> np.uint64(16) & np.uint64(0xFFFF)).astype(np.int64) << 4 | 8)


def decode(code, e, top):
    """top: 15 for m, 31 for v."""
    code, e = code.astype(np.int64), np.repeat(e.astype(np.int64), BLOCK)
    c = code & 127 if top == 15 else code
    q = np.where(c == 0, 0, np.maximum(c + 8 * (e - top), 0))
    x = np.where(e == 255, np.float32(np.nan), (q << 20).astype(np.uint32).view(np.float32))
    return np.where((code > 127) & (top == 15), -x, x).astype(np.float32)


def encode(x, d, top):
    bits = np.abs(x).view(np.uint32).astype(np.int64)
    e = (bits.reshape(-1, BLOCK).max(1) + (1 << 20)) >> 23
    off = 8 * (np.repeat(e, BLOCK) - top)
    q = (bits + d) >> 20
    if top == 15:
        c = np.where(bits == 0, 0, np.clip(q - off, 0, 127)) + 128 * (x < 0)
    else:
        c = np.where(bits == 0, 0, np.clip(np.maximum(q, 1) - off, 1, 255))
    return c.astype(np.uint8), e.astype(np.uint8)


def moments32(m, v, g, b1, b2):
    """The moments with every operation rounded to 32 bits (what 8-bit codes are made from)."""
    f = np.float32
    with np.errstate(all="ignore"):
        return f(b1) * m + f(1 - b1) * g, f(b2) * v + f(1 - b2) * (g * g)


# ------------------------------------------------------------------------------------------------------------- AdamW
def adamw(w, g, m, v, *, step, lr, b1, b2, eps, decay, horizon, w_half, hat_half, rounded=None):
    """64-bit step of one tensor and the bounds of a 32-bit one: (w, m, v, w_hat) and (bw, bm, bv, bhat).

    m: coefficient, product (twice) and sum: 4 roundings of each term; v: the square as well, and the gradient's scaling
    twice: 6.  The direction: the moments' errors, sqrt, the corrections, the sum with eps, the quotient and the product with
    lr, of one unit at most each: 16 half units, and half of v's relative error.  Weights: three more of what enters."""
    c1, c2 = 1 - b1 ** step, 1 - b2 ** step
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    bm = 5 * EPS * (np.abs(b1 * m) + np.abs((1 - b1) * g)) + TINY
    bv = 8 * EPS * v2 + TINY
    den = np.sqrt(v2 / c2) + eps
    d = lr * (m2 / c1) / den
    bd = lr / c1 * bm / den + np.abs(d) * (16 * EPS + 0.5 * bv / np.maximum(v2, TINY)) + TINY
    w2 = w - lr * decay * w - d
    hat = w2 - horizon * d
    bw = bd + 4 * EPS * (np.abs(w) * (1 + lr * abs(decay)) + np.abs(d))
    bh = bw + abs(horizon) * bd + 4 * EPS * (np.abs(w2) + abs(horizon) * np.abs(d))
    return (w2, m2, v2, hat), (bw + w_half * (np.abs(w2) + bw), bm, bv, bh + hat_half * (np.abs(hat) + bh))


# --------------------------------------------------------------------------------------------------- log probabilities
def log_probs(x, t, scale):
    """x [rows, vocab] in 64 bits: dict of logp, entropy, norm and the whole ln p, and bounds of a 32-bit evaluation.

    A scaled logit has 1 rounding, its distance d to the maximum 2 more of them and one of d; e^d that error and 4 units more
    (argument of the exponential in another base: 2 EPS |d|; the function: 2 units).  A sum of positive terms over vocab
    values in at least 64 chains: vocab / 64 + 16 roundings."""
    with np.errstate(all="ignore"):
        xs = scaled(x, scale)
        m = xs.max(1)
        empty = m == -np.inf
        ref = np.where(empty, 0, m)
        d = xs - ref[:, None]
        e = np.exp(d)
        s = np.where(empty, 1, e.sum(1))
        p = e / s[:, None]
        ls = np.where(empty, 0, np.log(s))
        lnp = d - ls[:, None]
        mean = (p * np.where(p > 0, d, 0)).sum(1)
        h = np.where(empty, 0, ls - mean)
        there = (t >= 0) & (t < x.shape[1])
        lt = lnp[np.arange(len(t)), np.where(there, t, 0)]
        logp = np.where(there, lt, 0)
        # the distance's error for each logit, and the relative error of its exponential
        fin = np.where(np.isfinite(d), np.abs(d), 0)
        de = EPS * (2 * np.where(np.isfinite(xs), np.abs(xs), 0) + 2 * np.abs(ref)[:, None] + fin)
        ee = de + EPS * (2 * fin + 8)
        depth = (x.shape[1] / 64 + 16) * EPS
        bls = (p * ee).sum(1) + depth + 4 * EPS * (1 + np.abs(ls))
        bh = bls + (p * (ee + depth) * fin + p * de).sum(1) + np.abs(mean) * ((p * ee).sum(1) + depth + 4 * EPS) + 4 * EPS * (np.abs(h) + np.abs(mean))
        bl = bls[:, None] + de + 4 * EPS * (np.abs(np.where(np.isfinite(lnp), lnp, 0)) + fin)
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -np.where(np.isnan(x), np.inf, x) , ~np.isnan(x)), axis=1)
    return dict(logp=logp, entropy=h, norm=np.stack([m, ls], 1), lnp=lnp, order=order,
                b_logp=np.where(there, bl[np.arange(len(t)), np.where(there, t, 0)], 0), b_entropy=bh, b_ls=bls,
                b_m=2 * EPS * np.abs(ref), b_lnp=bl)


def log_probs_grad(x, t, norm, entropy, gl, ge, scale, half):
    """The gradient in 64 bits from the norm and entropy that were handed over, and the bound of a 32-bit evaluation."""
    with np.errstate(all="ignore"):
        xs = scaled(x, scale)
        m, ls = norm[:, :1], norm[:, 1:]
        empty = m == -np.inf
        lnp = xs - np.where(empty, 0, m) - ls
        p = np.exp(lnp)
        there = (t >= 0) & (t < x.shape[1])
        one = np.zeros_like(p)
        one[np.arange(len(t))[there], t[there]] = 1
        g1 = np.where(there, gl, 0)[:, None]
        fin = np.where(np.isfinite(lnp), lnp, 0)
        d = g1 * (one - p)
        dl = EPS * (2 * np.where(np.isfinite(xs), np.abs(xs), 0) + 3 * np.abs(np.where(empty, 0, m)) + 3 * np.abs(ls) + 3 * np.abs(fin))
        pe = dl + EPS * (2 * np.abs(fin) + 10)
        b = np.abs(g1) * (p * pe + 4 * EPS * (one + p))
        if ge is not None:
            d = d - ge[:, None] * p * (fin + entropy[:, None])
            b = b + np.abs(ge)[:, None] * p * (np.abs(fin + entropy[:, None]) * (pe + 6 * EPS) + dl + 3 * EPS * (np.abs(fin) + np.abs(entropy)[:, None]))
        d = np.where(empty, 0, d * scale)
        b = scale * b + 4 * EPS * np.abs(d) + TINY * (1 + scale)
        return d, b + half * (np.abs(d) + b)


# ---------------------------------------------------------------------------------------------------------- embeddings
def embed_grad(g, ids, start, vocab, scale, add, half):
    """start: the table's gradient before; scale as a 32-bit number.  A row's sum of n terms: n roundings at most."""
    ids = ids.reshape(-1)
    there = (ids >= 0) & (ids < vocab)
    g = g.reshape(len(ids), -1)
    total, mag, n = np.zeros(start.shape), np.zeros(start.shape), np.zeros(vocab)
    np.add.at(total, ids[there], g[there])
    np.add.at(mag, ids[there], np.abs(g[there]))
    np.add.at(n, ids[there], 1)
    out = total * scale
    b = (n[:, None] + 3) * EPS * mag * abs(scale)
    if add:
        out = np.where(n[:, None] > 0, start + out, start)
        b = np.where(n[:, None] > 0, b + EPS * np.abs(out), 0)
    return out, np.where(n[:, None] > 0, b + half * (np.abs(out) + b) + TINY, 0)
