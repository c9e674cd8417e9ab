"""The operators between gather and reduction in 64 bits (numpy), written from their formulas, and what an implementation
in binary32 may be off by.

Every reference returns (value, size) for an output: `size` is what its terms add up to in magnitude, element by element,
so that a computation in binary32 is within `STEPS` * 2^-24 * size, and the stored result within half a unit in the last
place of its format of that.  STEPS counts the roundings on the way: a lane adds up to 64 numbers one after the other
(half of them matter on average, all of them at worst), a workgroup's tree and joins add some 30, exponentials and
reciprocal roots a few, and two nested sums meet in a norm's gradient.
"""
import numpy as np

STEPS = 160
U32 = 2.0 ** -24
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
# half of the smallest subnormal
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}


def within(got, value, size, fmt):
    """Whether `got` (float64) is a `fmt` rounding of something within the bound of `value`; infinities and NaN alike."""
    got, value = np.asarray(got, np.float64), np.asarray(value, np.float64)
    if fmt == "f16":
        value = np.where(np.abs(value) >= 65520, np.sign(value) * np.inf, value)       # rounds to infinity
    ok = np.isfinite(value)
    for alike in (np.isnan, np.isposinf, np.isneginf):
        if not np.array_equal(alike(got), alike(value)):
            return False
    size = np.broadcast_to(size, value.shape)
    tol = STEPS * U32 * size + HALF_ULP[fmt] * (np.abs(value) + STEPS * U32 * size) + TINY[fmt] + 2.0 ** -140
    return bool(np.all(np.abs(got - value)[ok] <= tol[ok]))


# ---- dropout -----------------------------------------------------------------------------------

def philox(block, seed):
    """Philox4x32-10 of 64-bit counters (the upper half of the counter 0): an array of four 32-bit words each."""
    block = np.asarray(block, np.uint64)
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    x = [block & low, block >> s, np.zeros_like(block), np.zeros_like(block)]
    return philox_words(x, seed)


def philox_words(x, seed):
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> s) ^ x[1] ^ np.uint64(k0), b & low, (a >> s) ^ x[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(x, -1)


def threshold(drop):
    return min(65535, int(np.rint(65536.0 * float(np.float32(drop)))))


def kept(rows, cols, drop, seed, offset):
    groups = -(-cols // 8)
    with np.errstate(over="ignore"):
        block = np.arange(rows * groups, dtype=np.uint64) + np.uint64(offset)
    words = philox(block, seed)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(rows, groups * 8)
    return halves[:, :cols] >= np.uint64(threshold(drop))


def dropped(v, drop, seed, offset):
    t = threshold(drop)
    if t == 0:
        return v
    return np.where(kept(*v.shape, drop, seed, offset), v * (65536.0 / (65536 - t)), 0.0)


def bias_dropout_add(x, bias, residual, drop, seed, offset):
    v = x if bias is None else x + bias
    size = np.abs(x) + (0 if bias is None else np.abs(bias))
    out = dropped(v, drop, seed, offset)
    size = dropped(size, drop, seed, offset)
    if residual is not None:
        out, size = out + residual, size + np.abs(residual)
    return out, size


def bias_dropout_add_backward(dout, drop, seed, offset):
    dx = dropped(dout, drop, seed, offset)
    return (dx, np.abs(dx)), (dx.sum(0), np.abs(dx).sum(0))


# ---- layer norm --------------------------------------------------------------------------------

def layer_norm(s, s_size, weight, bias, eps):
    """(y), (mean), (rstd), each with its size; s_size: that of s, where it is a computed value."""
    n = s.shape[1]
    weight = np.ones(n) if weight is None else weight
    bias = np.zeros(n) if bias is None else bias
    mean = s.mean(1)
    d = s - mean[:, None]
    var = (d * d).mean(1)
    with np.errstate(divide="ignore"):
        rstd = 1.0 / np.sqrt(var + eps)
    mean_size = s_size.mean(1)
    d_size = s_size + mean_size[:, None]
    # an error e of the variance moves rstd by e / (2 (var + eps)) of itself
    with np.errstate(divide="ignore", invalid="ignore"):
        relative = 1.0 + (d_size * np.abs(d)).mean(1) / (var + eps) + STEPS * U32 * (d_size * d_size).mean(1) / (var + eps)
    y = d * rstd[:, None] * weight + bias
    y_size = (d_size + np.abs(d) * relative[:, None]) * rstd[:, None] * np.abs(weight) + np.abs(bias)
    return (y, y_size), (mean, mean_size), (rstd, rstd * relative)


def layer_norm_backward(dy, x, mean, rstd, weight):
    """(dx), (dweight), (dbias) from the given statistics."""
    n = x.shape[1]
    weight = np.ones(n) if weight is None else weight
    rstd = rstd[:, None]
    hat = (x - mean[:, None]) * rstd
    hat_size = (np.abs(x) + np.abs(mean[:, None])) * rstd
    g = dy * weight
    c1, c2 = g.mean(1, keepdims=True), (g * hat).mean(1, keepdims=True)
    c1_size, c2_size = np.abs(g).mean(1, keepdims=True), (np.abs(g) * hat_size).mean(1, keepdims=True)
    dx = rstd * (g - c1 - hat * c2)
    dx_size = rstd * (np.abs(g) + c1_size + hat_size * c2_size)
    return (dx, dx_size), ((dy * hat).sum(0), (np.abs(dy) * hat_size).sum(0)), (dy.sum(0), np.abs(dy).sum(0))


def block_backward(dy, dsum, s, mean, rstd, weight, drop, seed, offset):
    """(dx), (dresidual), (dbias), (dweight), (dnorm_bias)."""
    (ds, size), dweight, dnorm_bias = layer_norm_backward(dy, s, mean, rstd, weight)
    if dsum is not None:
        ds, size = ds + dsum, size + np.abs(dsum)
    dx, dx_size = dropped(ds, drop, seed, offset), dropped(size, drop, seed, offset)
    return (dx, dx_size), (ds, size), (dx.sum(0), dx_size.sum(0)), dweight, dnorm_bias


# ---- log probabilities -------------------------------------------------------------------------

def logprobs(x, targets, top):
    """dict of logprob, entropy, lse (value, size), ids, top (value, size)."""
    rows, n = x.shape
    with np.errstate(all="ignore"):
        m = x.max(1)
        safe = np.where(np.isneginf(m), 0.0, m)
        e = np.exp(x - safe[:, None])
        z = e.sum(1)
        empty = z == 0
        logz = np.log(z)
        lse = np.where(empty, -np.inf, safe + logz)
        d = np.where(e == 0, 0.0, x - safe[:, None])
        far = (np.abs(d) * e).sum(1) / z
        entropy = np.where(empty, 0.0, logz - (d * e).sum(1) / z)
        logp = np.where(empty[:, None], -np.inf, x - lse[:, None])
        size = np.where(empty, 0.0, np.abs(safe) + np.abs(logz) + 1.0 + far)
        entropy_size = np.where(empty, 0.0, (np.abs(logz) + 1.0 + far) * (1.0 + far) + (d * d * e).sum(1) / z)
        at = np.clip(targets, 0, n - 1)
        of = np.where(targets < 0, 0.0, logp[np.arange(rows), at])
        of = np.where(targets >= n, np.nan, of)
    key = np.where(np.isnan(x), np.inf, x)
    # NaN before +inf before the numbers, the lower index first
    order = np.lexsort((np.broadcast_to(np.arange(n), x.shape), -key, ~np.isnan(x)), axis=1)[:, :top]
    best = np.take_along_axis(logp, order, 1)
    best_size = np.abs(np.where(np.isfinite(best), best, 0)) + size[:, None]
    of_size = np.where(targets < 0, 0.0, size + np.abs(np.where(np.isfinite(of), of, 0)))
    return dict(logprob=(of, of_size), entropy=(entropy, entropy_size), lse=(lse, size),
                ids=order, top=(best, best_size))


def logprobs_backward(x, targets, lse, entropy, dlogprob, dentropy):
    rows, n = x.shape
    g = np.where(targets < 0, 0.0, dlogprob)[:, None]
    h = (np.zeros(rows) if dentropy is None else dentropy)[:, None]
    with np.errstate(all="ignore"):
        logp = x - lse[:, None]
        p = np.exp(logp)
        plogp = np.where(p == 0, 0.0, p * (logp + (0 if dentropy is None else entropy[:, None])))
        hit = np.arange(n)[None, :] == targets[:, None]
        d = g * (hit - p) - h * plogp
        far = np.where(p == 0, 0.0, np.abs(x) + np.abs(lse[:, None]) + 1.0)
        ent = 0.0 if dentropy is None else np.abs(entropy)[:, None]
        # the exponential multiplies errors of its argument
        size = np.abs(g) * (hit + p * far) + np.abs(h) * p * (far + ent) * far
    none = ((g == 0) & (h == 0))[:, 0] | np.isneginf(lse)
    d[none], size[none] = 0.0, 0.0
    d[targets >= n] = np.nan
    return d, size
