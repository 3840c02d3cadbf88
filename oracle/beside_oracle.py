"""fp64 NumPy reference of what stands beside the losses: e4m3 in blocks, top logits, sampling, the norm of the gradients.
Shares no code with the GPU path."""
import numpy as np

MAX = 448.0
LEAST = 448 * 2.0 ** -126


def e4m3(v):
    """Nearest e4m3 value, ties to the even code, magnitudes beyond 448 to 448."""
    v = np.asarray(v, np.float64)
    a = np.abs(v)
    e = np.frexp(np.maximum(a, 2.0 ** -6))[1] - 1                  # a in [2^e, 2^(e+1)), or below the smallest normal
    unit = np.ldexp(1.0, e - 3)
    return np.copysign(np.minimum(np.rint(a / unit) * unit, MAX), v)


def blocks(x, tile):
    """(values of the codes, scales) of [R, C], a scale per row and 128 columns or per 128 x 128; both in fp64, the scale rounded to
    fp32 as it is kept."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    high = 128 if tile else 1
    codes = np.zeros_like(x)
    scales = np.zeros((-(-R // high), -(-C // 128)))
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            at = (slice(i * high, (i + 1) * high), slice(j * 128, (j + 1) * 128))
            m = max(np.abs(x[at]).max(), LEAST)
            codes[at] = e4m3(x[at] * MAX / m)
            scales[i, j] = np.float32(m / MAX)
    return codes, scales


def expand(scales, R, C, tile):
    s = np.repeat(scales, 128, 1)[:, :C]
    return np.repeat(s, 128, 0)[:R] if tile else s


def top_logits(z, K, tau):
    """(logits, indices, lse): descending, ties to the lower index; minus infinity is no entry."""
    z = np.asarray(z, np.float64)
    T = z.shape[0]
    top, index = np.full((T, K), -np.inf), np.full((T, K), -1, np.int64)
    for t in range(T):
        order = np.lexsort((np.arange(z.shape[1]), np.where(np.isnan(z[t]), -np.inf, -z[t])))[:K]
        there = ~(z[t][order] == -np.inf)
        top[t, :there.sum()], index[t, :there.sum()] = z[t][order][there], order[there]
    with np.errstate(invalid="ignore", divide="ignore"):
        y = z / tau
        m = y.max(1, keepdims=True)
        lse = np.where(np.isfinite(m[:, 0]), (m + np.log(np.exp(y - np.where(np.isfinite(m), m, 0)).sum(1, keepdims=True)))[:, 0], m[:, 0])
    return top, index, lse


def kept(z, temperature, top_k, top_p, min_p):
    """(indices that are kept, in ascending order; their weights) of one row."""
    order = np.lexsort((np.arange(z.size), -z))
    w = np.exp((z[order] - z[order[0]]) / temperature)
    n = z.size if top_k == 0 else min(top_k, z.size)
    run = np.cumsum(w[:n])
    if top_p < 1:
        n = 1 + int((run[:-1] < top_p * run[-1]).sum())
    n = int((w[:n] >= min_p).sum())
    ids = order[:n]
    back = np.argsort(ids)
    return ids[back], w[:n][back]


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability) of one row; settings as the 32-bit numbers that are passed."""
    z, u = np.asarray(z, np.float64), float(np.float32(u))
    temperature, top_p, min_p = (float(np.float32(v)) for v in (temperature, top_p, min_p))
    top = z.max()
    if not np.isfinite(top) or np.isnan(z).any() or not 0 <= u < 1:
        return -1, np.nan
    if temperature == 0:
        return int(np.argmax(z)), 0.0
    ids, w = kept(z, temperature, top_k, top_p, min_p)
    run = np.cumsum(w)
    at = int(np.searchsorted(run, u * run[-1], side="right"))
    return int(ids[at]), float(np.log(w[at] / run[-1]))


def distance(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """How far u, top_p and min_p are from the next value at which another token would come out, relative to the sums they are compared
    with: a result is only pinned where this is more than the sums' error."""
    z = np.asarray(z, np.float64)
    temperature, top_p, min_p = (float(np.float32(v)) for v in (temperature, top_p, min_p))
    if temperature == 0:
        return 1.0
    order = np.lexsort((np.arange(z.size), -z))
    w = np.exp((z[order] - z[order[0]]) / temperature)[:z.size if top_k == 0 else top_k]
    run = np.cumsum(w)
    d = [1.0]
    if top_p < 1:
        d.append(np.abs(run / run[-1] - top_p).min())
    if min_p > 0:
        x = np.abs(w[1:] - min_p)
        d.append(x.min() if x.size else 1.0)
    _, wk = kept(z, temperature, top_k, top_p, min_p)
    run = np.cumsum(wk)
    d.append(np.abs(run[:-1] / run[-1] - float(np.float32(u))).min() if run.size > 1 else 1.0)
    return min(d)


def clip(grads, max_norm, largest=False):
    """(norm, clipped gradients)."""
    g = [np.asarray(x, np.float64) for x in grads]
    norm = max([np.abs(x).max() for x in g if x.size], default=0.0) if largest else np.sqrt(sum((x ** 2).sum() for x in g))
    f = min(1.0, max_norm / norm) if norm > 0 and np.isfinite(norm) else 1.0
    return norm, [x * f for x in g]
