"""Float64 checker of what follows a step's gradients and of the loss on pairs of rollouts: preference loss, gradient norm, AdamW step, moments
in 8 bits.  Plain loops by the definitions; shares no code with the product.  The codes of 8-bit moments are defined by single
roundings in float32, which numpy reproduces."""
import math

import numpy as np

from .drafter_oracle import MASKED, log_partition

LOGISTIC, HINGE, SQUARE = 0, 1, 2


def softplus(x):
    return max(x, 0.0) + math.log1p(math.exp(-abs(x))) if math.isfinite(x) else (x if x > 0 else 0.0 if x < 0 else x)


def pair_value(kind, x, beta, smoothing):
    if kind == HINGE:
        return max(0.0, 1.0 - x) if x == x else x
    if kind == SQUARE:
        return ((x - 0.5) / beta) ** 2
    up = softplus(x) if smoothing else 0.0
    return (1 - smoothing) * softplus(-x) + smoothing * up


def pair_slope(kind, x, beta, smoothing):
    if x != x:
        return x
    if kind == HINGE:
        return -1.0 if x < 1.0 else 0.0
    if kind == SQUARE:
        return 2 * (x - 0.5) / beta ** 2
    sigma = lambda y: 1 / (1 + math.exp(-y)) if y > -700 else 0.0   # noqa: E731
    return -(1 - smoothing) * sigma(-x) + smoothing * sigma(x)


def preference(logprob, ref, rollout, R, chosen, rejected, weight, kind=LOGISTIC, average=0, beta=0.1, smoothing=0.0, margin=0.0):
    """loss, margins [P], ratios [R], slopes [R] (dloss / dratio, with `average` over the number of tokens), numbers of tokens [R]."""
    total, count = np.zeros(R), np.zeros(R, np.int64)
    for t in range(len(rollout)):
        r = rollout[t]
        if 0 <= r < R:
            total[r] += logprob[t] - (ref[t] if ref is not None else 0.0)
            count[r] += 1
    if average:
        total = total / np.maximum(count, 1)
    loss, m, slope = 0.0, np.zeros(len(chosen)), np.zeros(R)
    for p in range(len(chosen)):
        c, j = chosen[p], rejected[p]
        w = float(weight[p]) if weight is not None else 1.0 / len(chosen)
        if not (0 <= c < R and 0 <= j < R) or w == 0.0:
            continue
        m[p] = beta * (total[c] - total[j])
        loss += w * pair_value(kind, m[p] - margin, beta, smoothing)
        s = beta * w * pair_slope(kind, m[p] - margin, beta, smoothing)
        slope[c] += s
        slope[j] -= s
    if average:
        slope = slope / np.maximum(count, 1)
    return loss, m, total, slope, count


def preference_rows(z, V, targets, ref, rollout, R, chosen, rejected, weight, grad_scale=1.0, **how):
    """The same from logits: loss, margins, ratios, slopes, logprob [T], dlogits [T, V], q [T, V]."""
    T = len(z)
    lp, part = np.zeros(T), np.array(rollout, np.int64)
    for t in range(T):
        row = np.asarray(z[t][:V], np.float64)
        if not (0 <= rollout[t] < R and 0 <= targets[t] < V):
            part[t] = -1
            continue
        lse = log_partition(row)
        if lse == -np.inf:
            part[t] = -1
        elif lse != lse:
            lp[t] = np.nan
        else:
            lp[t] = row[targets[t]] - lse if row[targets[t]] > MASKED else -np.inf
    loss, m, total, slope, _ = preference(lp, ref, part, R, chosen, rejected, weight, **how)
    dz, q = np.zeros((T, V)), np.zeros((T, V))
    for t in range(T):
        if part[t] < 0 or slope[part[t]] == 0.0:
            continue
        row = np.asarray(z[t][:V], np.float64)
        lse = log_partition(row)
        q[t] = np.where(row > MASKED, np.exp(np.where(row > MASKED, row, 0.0) - lse), 0.0) if lse == lse else np.nan
        dz[t] = -slope[part[t]] * grad_scale * q[t]
        dz[t][targets[t]] += slope[part[t]] * grad_scale
    return loss, m, total, slope, lp, dz, q


# ------------------------------------------------------------------------------------------------ AdamW
F = np.float32
BLOCK, TOP1, TOP2 = 256, F(127 ** 2), F(255 ** 4)


def mix(x):
    x = np.asarray(x, np.uint64) & 0xffffffff
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xffffffff
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xffffffff
    return x ^ (x >> 16)


def random_bits(seed, steps_before, tensor, n):
    of_step = mix((seed & 0xffffffff) ^ int(mix((seed >> 32) ^ int(mix(steps_before)))))
    return mix(int(mix(int(of_step) + tensor)) + np.arange(n, dtype=np.uint64))


def scale_of(x, top):
    """One scale for each block of 256 of x."""
    out = np.zeros((len(x) + BLOCK - 1) // BLOCK, F)
    for b in range(len(out)):
        block = np.abs(x[b * BLOCK:(b + 1) * BLOCK])
        s = block.max() * F(1.0 / float(top))
        out[b] = np.nan if not np.isfinite(block).all() else s if s >= np.finfo(F).tiny else 0.0
    return out


def codes_of(x, scale, u, first):
    """Codes (whole numbers) of x [n] f32 with the scales of its blocks; u [n] in (0, 1)."""
    s = np.repeat(scale, BLOCK)[:len(x)]
    power = (lambda c: c * c) if first else (lambda c: (c * c) * (c * c))
    top = TOP1 if first else TOP2
    with np.errstate(all="ignore"):
        y = np.minimum(np.abs(x) * (F(1) / s), top)
    y = np.where(s > 0, y, F(0)).astype(F)
    grid = power(np.arange(257, dtype=F))
    c = np.searchsorted(grid, y, side="right") - 1
    c = np.clip(c, 0, 127 if first else 255)
    step = (u.astype(F) * ((F(2) * c.astype(F) + F(1)) if first else (grid[c + 1] - grid[c]))).astype(F)
    c = c + (step < y - grid[c])
    c = np.clip(c, 0, 127 if first else 255)
    if first:
        return np.where(x < 0, -c, c)
    return np.where((y > 0) & (c < 1), 1, c)


def values_of(codes, scale, first):
    c = codes.astype(F)
    s = np.repeat(scale, BLOCK)[:len(codes)]
    return ((c * np.abs(c)) * s if first else ((c * c) * (c * c)) * s).astype(F)


def moments32(m, v, grad, factor, beta1, beta2):
    """Both moments as float32 forms them, each product and sum rounded by itself."""
    with np.errstate(all="ignore"):
        g = (grad.astype(F) * F(factor)).astype(F)
        m = (m * F(beta1)).astype(F) + (g * F(1 - beta1)).astype(F)
        v = (v * F(beta2)).astype(F) + ((g * g).astype(F) * F(1 - beta2)).astype(F)
    return m.astype(F), v.astype(F)


def adamw(p, m, v, grad, steps_before, lr, beta1, beta2, eps, weight_decay, factor=1.0, decay=1.0):
    """One step in 64 bits: new p, m, v."""
    t = steps_before + 1
    g = np.float64(factor) * grad
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p - lr * (decay * weight_decay * p + step), m, v
