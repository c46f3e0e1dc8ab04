"""Plain 64-bit (numpy) implementations of the norm, of 8-bit microscaled rows, of scores from
them and of the cross entropy over a table, written from their formulas and sharing no
code with the library."""
import numpy as np


def e4m3_values():
    """The value of every E4M3 code (127 and 255 are NaN)."""
    v = np.empty(256)
    for c in range(128):
        e, m = c >> 3, c & 7
        v[c] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    v[127] = np.nan
    v[128:] = -v[:128]
    return v


E4M3 = e4m3_values()


def quantize8(y):
    """(codes, scales) of y [rows, dim]: blocks of 32, the smallest power of two that keeps a
    block within 448, the nearest code, ties to the even one."""
    rows, dim = y.shape
    groups = -(-dim // 128)
    codes = np.zeros((rows, groups * 128), np.uint8)
    scales = np.zeros((rows, groups * 4), np.uint8)
    pos = E4M3[:127]
    for r in range(rows):
        for b in range(-(-dim // 32)):
            v = y[r, b * 32:(b + 1) * 32]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            top = np.abs(v).max()
            e = -127
            if top > 0:
                e = max(int(np.floor(np.log2(top))) - 9, -127)
                while top > 448.0 * 2.0 ** e:
                    e += 1
                scales[r, b] = e + 127
            a = np.abs(v) * 2.0 ** -e
            i = np.searchsorted(pos, a).clip(1, 126)  # pos[i - 1] < a <= pos[i]
            lo, hi = a - pos[i - 1], pos[i] - a
            c = np.where((lo < hi) | ((lo == hi) & (i % 2 == 1)), i - 1, i)
            codes[r, b * 32:b * 32 + v.size] = c + 128 * np.signbit(v)
    return codes, scales


def values8(codes, scales, dim):
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    v = E4M3[codes].reshape(codes.shape[0], -1, 32) * s[:, :, None]
    return v.reshape(codes.shape[0], -1)[:, :dim]


def rmsnorm(h, w, eps):
    """(y, n = h / rms, rms): y = n w."""
    rms = np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h / rms * w, h / rms, rms


def rmsnorm_grad(dy, h, w, eps, dsum=0.0):
    """(dh, dw) and the magnitudes that their rounding errors are relative to."""
    _, n, rms = rmsnorm(h, w, eps)
    g = dy * w
    mean = (n * g).mean(1, keepdims=True)
    dh = (g - n * mean) / rms + dsum
    size = (np.abs(g) + np.abs(n) * np.abs(n * g).mean(1, keepdims=True)) / rms + np.abs(dsum)
    return dh, (dy * n).sum(0), size, np.abs(dy * n).sum(0)


def xent(x, w, labels, weights=None, scale=1.0):
    """loss, dx, dw, and p - onehot (all rows' weights in dx and dw); rows with a negative label
    are left out."""
    N, V = x.shape[0], w.shape[0]
    weights = np.ones(N) if weights is None else weights
    live = (labels >= 0) & (weights != 0)
    loss, dx = np.zeros(N), np.zeros(x.shape)
    d = np.zeros((N, V))
    z = scale * (x[live] @ w.T)
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    total = e.sum(1, keepdims=True)
    i = np.arange(z.shape[0])
    loss[live] = weights[live] * (np.log(total[:, 0]) + top[:, 0] - z[i, labels[live]])
    p = e / total
    p[i, labels[live]] -= 1.0
    d[live] = p
    dx[live] = scale * weights[live, None] * (p @ w)
    dw = scale * (p * weights[live, None]).T @ x[live]
    return loss, dx, dw, d
