"""Plain 64-bit (numpy) implementations of the output head's operators, written
from their formulas and sharing no code with the library."""
import math

import numpy as np

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
VALUES = np.array(GRID + [-v for v in GRID])


def blocks(dim):
    return -(-dim // 32)


def bf16_round(x):
    """float64 -> the nearest BF16 value, ties to even, as float64.  The values
    given here are FP32 numbers or sums whose second rounding does not matter."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    r = np.where(np.isnan(x), np.uint32(0x7FC00000), r)
    return r.view(np.float32).astype(np.float64)


def quantize(x):
    """(codes, scales) of x [rows, dim], element by element."""
    rows, dim = x.shape
    nb = blocks(dim)
    codes = np.zeros((rows, nb * 16), np.uint8)
    scales = np.zeros((rows, -(-nb // 4) * 4), np.uint8)
    for r in range(rows):
        for b in range(nb):
            v = [float(t) for t in x[r, b * 32:(b + 1) * 32]]
            if not all(math.isfinite(t) for t in v):
                scales[r, b] = 255
                continue
            top = max(abs(t) for t in v)
            e = -127 if top == 0 else max(math.frexp(top)[1] - 1 - 2, -127)
            scales[r, b] = e + 127
            for i, t in enumerate(v):
                y = abs(t) * 2.0 ** -e
                best = min(range(8), key=lambda c: (abs(min(y, 6.0) - GRID[c]), c % 2))
                if math.copysign(1.0, t) < 0:
                    best += 8
                codes[r, b * 16 + i // 2] |= best << (4 * (i % 2))
    return codes, scales


def dequantize(codes, scales, dim):
    rows = codes.shape[0]
    v = np.empty((rows, codes.shape[1] * 2))
    v[:, 0::2] = VALUES[codes & 15]
    v[:, 1::2] = VALUES[codes >> 4]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v.reshape(rows, -1, 32) * s[:, :blocks(dim), None]).reshape(rows, -1)[:, :dim]


def pooled(tables, batch, indices, offsets, weights=None, mean=False):
    """Bags of float64 tables, and the sums of the terms' magnitudes."""
    T, dim = len(tables), tables[0].shape[1]
    y = np.zeros((T, batch, dim))
    mag = np.zeros((T, batch, dim))
    for t in range(T):
        for b in range(batch):
            k = t * batch + b
            for s in range(offsets[k], offsets[k + 1]):
                v = tables[t][indices[s]] * (1.0 if weights is None else float(weights[s]))
                y[t, b] += v
                mag[t, b] += np.abs(v)
            n = offsets[k + 1] - offsets[k]
            if mean and n:
                y[t, b] /= n
                mag[t, b] /= n
    return y, mag


def logits(x, seen=None, prompt_lens=None, repetition=None, frequency=None, presence=None,
           bias=None, masks=None, mask_ids=None):
    """Rows after penalties, biases and masks; seen: a list of tokens per row,
    bias: a list of (id, value) per row.  Also the magnitudes that roundings
    are relative to."""
    y = np.array(x, np.float64)
    mag = np.zeros_like(y)
    rows, vocab = y.shape
    one = lambda a, r, d: d if a is None else float(a[r])
    with np.errstate(invalid="ignore"):
        for r in range(rows):
            if seen is not None:
                n = 0 if prompt_lens is None else int(prompt_lens[r])
                rho = one(repetition, r, 1.0)
                for v in set(seen[r]):
                    y[r, v] = y[r, v] / rho if y[r, v] > 0 else y[r, v] * rho
                    c = list(seen[r][max(n, 0):]).count(v)
                    if c:
                        pen = one(frequency, r, 0.0) * c + one(presence, r, 0.0)
                        mag[r, v] += 3 * (abs(one(frequency, r, 0.0) * c) + abs(one(presence, r, 0.0)))
                        y[r, v] -= pen
                    mag[r, v] += 3 * abs(y[r, v])
            if bias is not None:
                for v, value in dict(bias[r]).items():
                    mag[r, v] += abs(y[r, v])
                    y[r, v] += float(value)
                    mag[r, v] += abs(y[r, v])
            if masks is not None:
                m = r if mask_ids is None else int(mask_ids[r])
                if m >= 0:
                    for v in range(vocab):
                        if not (int(masks[m][v // 32]) >> (v % 32)) & 1:
                            y[r, v], mag[r, v] = -np.inf, 0.0
    return y, mag


def distill(x, ids, teacher, temperature, weights=None):
    """(loss, grad, q, sum of |terms| of the loss) per row."""
    x = np.asarray(x, np.float64)
    rows, vocab = x.shape
    T = float(temperature)
    loss, grad, prob = np.zeros(rows), np.zeros((rows, vocab)), np.zeros((rows, vocab))
    mag = np.zeros(rows)
    with np.errstate(invalid="ignore", over="ignore"):
        for r in range(rows):
            w = 1.0 if weights is None else float(weights[r])
            entries = [(int(i), float(t) / T) for i, t in zip(ids[r], teacher[r]) if i >= 0]
            if w == 0 or all(t == -np.inf for _, t in entries) or np.all(x[r] == -np.inf):
                continue
            top = max(t for _, t in entries)
            e = [np.exp(t - top) for _, t in entries]
            p = [v / sum(e) for v in e]
            z = x[r] / T
            ref = np.max(z[~np.isnan(z)]) if not np.all(np.isnan(z)) else 0.0
            ex = np.exp(z - ref)
            total = ex.sum()
            q = ex / total
            lse = ref + np.log(total)
            grad[r] = q
            for (v, t), pk in zip(entries, p):
                if pk > 0 or np.isnan(pk):
                    logp = t - top - np.log(sum(e))
                    loss[r] += pk * (logp - (z[v] - lse))
                    mag[r] += pk * (abs(logp) + abs(z[v]) + abs(lse)) if np.isfinite(z[v]) else 0
                    grad[r, v] -= pk
            loss[r] *= w * T * T
            mag[r] *= abs(w) * T * T
            grad[r] *= w * T
            prob[r] = q
    return loss, grad, prob, mag
