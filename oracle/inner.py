"""CPU oracle of the inner step's operators -- TEST INFRASTRUCTURE, same rules as the rest of oracle/.

    norm     n = sqrt(sum g^2), factor = min(1, max_norm / n), NaN where n is not finite
    AdamW    g = s grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
             theta = theta (1 - lr wd decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
    8 bits   blocks of 256 elements: e4m3 numbers times largest / 448, rounded by a threshold (see held())
    lookup   out[r] = scale (T[x_r] + P[x_r]) + pos[r mod L], one fp32 rounding per operation
    grad     G[x] = scale sum_{r: x_r = x} dY[r]

Plain numpy in float64 (the lookup, whose result is defined to the bit, in float32), the definitions written out; beside
each result the size of the terms it is made of, from which the tests derive how far fp32 may be off.
"""
from __future__ import annotations

import numpy as np

BLOCK = 256


def norm(grads, max_norm):
    with np.errstate(over="ignore", invalid="ignore"):
        n = float(np.sqrt(sum(float(np.sum(np.square(g.astype(np.float64)))) for g in grads)))
    if not np.isfinite(n):
        return n, float("nan")
    return n, (max_norm / n if n > max_norm else 1.0)


def adamw(theta, grad, m, root, *, lr, beta1, beta2, eps, weight_decay, step, scale=1.0, decay=1.0):
    """theta, grad, m and root = sqrt(v) before the step, float64.  Returns new theta, m, v and the bars of each per unit
    roundoff: how many roundings of which terms go into it."""
    g = scale * grad
    m_new = beta1 * m + (1 - beta1) * g
    v_new = beta2 * root * root + (1 - beta2) * g * g
    size = lr / (1 - beta1 ** step)
    below = np.sqrt(v_new / (1 - beta2 ** step)) + eps
    change = size * m_new / below
    theta_new = theta * (1 - lr * weight_decay * decay) - change
    # each term: its constant, the product(s) and the sum it enters, with the factor on the gradient (twice in g^2)
    bar_m = 5 * (np.abs(beta1 * m) + np.abs((1 - beta1) * g))
    bar_v = 7 * v_new
    # numerator; root (half of v's, and its own), its factor, eps, the sum, the quotient, the factor of size and the last difference
    bar_change = size * bar_m / below + (3.5 + 10) * np.abs(change)
    bar_theta = 5 * np.abs(theta) + bar_change + np.abs(theta_new)
    return theta_new, m_new, v_new, bar_theta, bar_m, bar_v


def thresholds(places, step, second):
    """t of the rounding rule as 20-bit fractions: multiples of 1/q and 1/q^2, q^3 = q + 1, in 32-bit fixed point."""
    word = (np.asarray(places, np.uint64) * np.uint64(0xC13FA9A9) + np.uint64((step * 0x91E10DA5 + (2 ** 31 if second else 0)) % 2 ** 32))
    return ((word % np.uint64(2 ** 32)) >> np.uint64(12)).astype(np.float64) / 2.0 ** 20


def held(x, places, step, second):
    """Values of whole blocks (x: [blocks, 256]) in 8 bits.  Returns (numbers, scales, edge): numbers * scales is what is
    held, edge how near, in gaps, each value lies to the point where its rounding changes."""
    most = np.abs(x).max(axis=1)
    scales = most / 448.0
    safe = np.where(scales > 0, scales, 1.0)
    a = np.abs(x) / safe[:, None]
    exponent = np.maximum(np.frexp(a)[1] - 1, -6)            # (frexp: a = f 2^e, 1/2 <= f < 1)
    gap = np.ldexp(1.0, exponent - 3)
    at = a / gap + thresholds(places, step, second).reshape(x.shape)
    numbers = np.minimum(np.floor(at) * gap, 448.0)
    if second:
        numbers = np.where((a > 0) & (numbers == 0), 2.0 ** -9, numbers)
    return numbers * np.sign(x), scales, np.abs(at - np.rint(at))


def lookup(table, ids, t_perp=None, pos=None, scale=1.0):
    """All float32."""
    at = np.clip(ids, 0, len(table) - 1)
    x = table[at]
    if t_perp is not None:
        x = x + t_perp[at]
    x = x * np.float32(scale)
    if pos is not None:
        x = x + pos[np.arange(len(ids)) % len(pos)]
    return x


def embedding_grad(grad_out, ids, vocab, scale, ignore_id=-1):
    """Returns the gradient, the sum of the magnitudes it is made of, and the number of tokens of each row."""
    keep = np.ones(len(ids), bool) if ignore_id < 0 else ids != ignore_id
    at = np.clip(ids, 0, vocab - 1)[keep]
    rows = float(np.float32(scale)) * grad_out[keep].astype(np.float64)
    total, size = np.zeros((vocab, grad_out.shape[1])), np.zeros((vocab, grad_out.shape[1]))
    np.add.at(total, at, rows)
    np.add.at(size, at, np.abs(rows))
    return total, size, np.bincount(at, minlength=vocab)
