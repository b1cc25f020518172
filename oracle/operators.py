"""Layer norm, log probabilities and AdamW in numpy float64, straight from their formulas: the reference of the operators around
the layers.  Tensors are [positions, C]; the 8-bit states are evaluated in float32, operation by operation, because which of
two neighbouring values a state takes is decided there."""
import numpy as np

F = np.float32


def norm_fwd(x, w=None, b=None, eps=1e-5):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    return (y if w is None else y * w + b), mean, rstd


def norm_bwd(x, w, g, mean, rstd):
    """From the mean and rstd that the backward pass is given."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None]
    xh = (x - np.asarray(mean, np.float64)[:, None]) * rstd
    h = g if w is None else g * w
    gx = rstd * (h - h.mean(1, keepdims=True) - xh * (h * xh).mean(1, keepdims=True))
    return gx, (g * xh).sum(0), g.sum(0)


def logp_fwd(x, target=None, top=0):
    """(logp, entropy, lse, top_logp, top_class) of scores x [positions, C]; -inf: masked; ignored positions as the library has them."""
    x = np.asarray(x, np.float64)
    rows, C = x.shape
    logp, entropy, lse = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    top_logp, top_class = np.full((rows, top), -np.inf), np.full((rows, top), -1, np.int32)
    for i in range(rows):
        t = None if target is None else int(target[i])
        if t is not None and not 0 <= t < C:
            continue
        live = np.flatnonzero(x[i] > -np.inf)
        if live.size == 0:
            logp[i] = lse[i] = -np.inf
            continue
        v = x[i, live]
        m = v.max()
        p = np.exp(v - m)
        lse[i] = m + np.log(p.sum())
        p /= p.sum()
        entropy[i] = -(p * (v - lse[i])).sum()
        if t is not None:
            logp[i] = x[i, t] - lse[i]
        best = live[np.lexsort((live, -v))[:top]]
        top_logp[i, :best.size], top_class[i, :best.size] = x[i, best] - lse[i], best
    return logp, entropy, lse, top_logp, top_class


def logp_bwd(x, target, lse, entropy, grad_logp=None, grad_entropy=None):
    x, lse = np.asarray(x, np.float64), np.asarray(lse, np.float64)
    rows, C = x.shape
    gx = np.zeros((rows, C))
    for i in range(rows):
        t = None if target is None else int(target[i])
        if (t is not None and not 0 <= t < C) or lse[i] == -np.inf:
            continue
        live = x[i] > -np.inf
        lp = x[i, live] - lse[i]
        if grad_logp is not None:
            gx[i, live] -= grad_logp[i] * np.exp(lp)
            gx[i, t] += grad_logp[i]
        if grad_entropy is not None:
            gx[i, live] -= grad_entropy[i] * np.exp(lp) * (lp + entropy[i])
    return gx


def adamw(p, m, v, g, t, lr, beta1, beta2, eps, decay):
    """Step t on float64 copies: (p, m, v)."""
    p, m, v, g = (np.asarray(a, np.float64) for a in (p, m, v, g))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps), m, v


# ---- states in 8 bits --------------------------------------------------------------------------------------------------

def mix(x):
    x = np.asarray(x, np.uint64) & np.uint64(0xFFFFFFFF)
    x = (x ^ x >> np.uint64(16)) * np.uint64(0x6A09E667) & np.uint64(0xFFFFFFFF)
    x = (x ^ x >> np.uint64(15)) * np.uint64(0xBB67AE85) & np.uint64(0xFFFFFFFF)
    return x ^ x >> np.uint64(16)


def noise(n, seed, t, tensor):
    """Two numbers in [0,1) for every element of a tensor in step t."""
    key = int(mix((int(mix(seed + t)) + tensor) & 0xFFFFFFFF))
    x = mix(np.arange(n, dtype=np.uint64) + np.uint64(key))
    return (x & np.uint64(0xFFFF)).astype(F) / F(65536), (x >> np.uint64(16)).astype(F) / F(65536)


def e4m3(codes):
    """The value of every e4m3 byte."""
    codes = np.asarray(codes, np.int64)
    e, f = codes >> 3 & 15, codes & 7
    value = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where(codes & 127 == 127, np.nan, np.where(codes >> 7 == 1, -value, value))


def widen(codes, scale):
    """fp32 values of a state: e4m3 bytes [n], e8m0 bytes [ceil(n/32)]."""
    return (e4m3(codes) * np.repeat(2.0 ** (np.asarray(scale, np.float64) - 127), 32)[:len(codes)]).astype(F)


def _blocks(x):
    return np.pad(x, (0, -len(x) % 32)).reshape(-1, 32)


def _exponent(x):
    return (x.view(np.int32) >> 23 & 255) - 127


def _block_exponent(x):
    bits = x.max(1).view(np.int32)
    return np.clip((bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000), -100, 120)


def _power(e):
    return np.ldexp(F(1), e).astype(F)


def store(x, r, root=None):
    """Codes and block exponents of a first moment x, or, with its root, of a second moment, rounded by r."""
    n, size = len(x), _blocks(np.abs(x) if root is None else root)
    x, r = _blocks(x), _blocks(r)
    e = _block_exponent(size)
    y = size * _power(-e)[:, None]
    ey = np.maximum(_exponent(y), -6)
    f = _power(3 - ey)
    if root is None:
        steps = np.floor((y * f).astype(np.float64) + r)      # (the sum not rounded)
    else:
        steps = np.floor(y * f)
        f = f * _power(-e)[:, None]
        w = x * f * f
        steps = steps + (r * (F(2) * steps + F(1)) < w - steps * steps)
        steps = np.where(x > 0, np.maximum(steps, 1), steps)
    codes = np.minimum((ey + 6) * 8 + steps.astype(np.int64), 126)
    if root is None:
        codes = codes | np.signbit(x).astype(np.int64) << 7
    return codes.reshape(-1)[:n].astype(np.uint8), (e + 127).astype(np.uint8)


def adamw_8bit(p, m, m_scale, v, v_scale, g, t, lr, beta1, beta2, eps, decay, seed, tensor, grad_scale=1.0):
    """Step t in float32, each operation rounded: (p before rounding to its type, m codes, m scales, v codes, v scales)."""
    g = np.asarray(g, F) * F(grad_scale)
    first = widen(m, m_scale) * F(beta1) + g * F(1 - beta1)
    root = widen(v, v_scale)
    second = root * root * F(beta2) + g * g * F(1 - beta2)
    root = np.sqrt(second)
    by = first / (root * F(1 / np.sqrt(1 - beta2 ** t)) + F(eps))
    p = np.asarray(p, F) * F(1 - lr * decay) - by * F(lr / (1 - beta1 ** t))
    r, r2 = noise(len(g), seed, t, tensor)
    return (p,) + store(first, r) + store(second, r2, root)
