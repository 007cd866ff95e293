"""Microscaled records in numpy and the distillation loss in 64 bits: the
plain definitions that the GPU tests compare with."""
import numpy as np

FP4 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6], np.float64)
FP8 = np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
                for e in range(16) for m in range(8)][:127], np.float64)   # code 127 is not a number


def record_bytes(dim, bits):
    nb = (dim + 31) // 32
    return (nb * (4 * bits + 1) + 15) // 16 * 16


def scale_of(code):
    return np.where(code == 255, np.nan, np.ldexp(1.0, code.astype(np.int64) - 127))


def scale_code(top, bits):
    """The scale byte of blocks whose largest magnitudes (fp32) are `top`."""
    field = top.astype(np.float32).view(np.uint32) >> 23
    return np.where(field == 255, 255, np.maximum(field.astype(np.int64) - (2 if bits == 4 else 8), 0))


def nearest(m, grid):
    """The grid's index nearest to each m >= 0, ties to the even index."""
    hi = np.clip(np.searchsorted(grid, m), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = m - grid[lo], grid[hi] - m
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(up, hi, lo)


def quantise(x, bits):
    """The records of the rows of x (any float array, its values in fp32)."""
    x = np.asarray(x, np.float32)
    n, dim = x.shape
    nb = (dim + 31) // 32
    v = np.zeros((n, nb * 32), np.float32)
    v[:, :dim] = x
    v = v.reshape(n, nb, 32)
    with np.errstate(invalid="ignore"):
        bits32 = (np.abs(v).view(np.uint32)).max(axis=2)
    code = scale_code(bits32.view(np.float32), bits)
    grid = FP4 if bits == 4 else FP8
    bad = code == 255
    m = np.abs(v.astype(np.float64)) / np.where(bad, 1.0, scale_of(np.where(bad, 127, code)))[:, :, None]
    q = nearest(np.where(bad[:, :, None], 0.0, m), grid).astype(np.uint8)
    sign = np.signbit(v) & ~bad[:, :, None]
    out = np.zeros((n, record_bytes(dim, bits)), np.uint8)
    if bits == 4:
        q = q | (sign.astype(np.uint8) << 3)
        out[:, :nb * 16] = (q[:, :, 0::2] | (q[:, :, 1::2] << 4)).reshape(n, nb * 16)
        out[:, nb * 16:nb * 17] = code
    else:
        out[:, :nb * 32] = (q | (sign.astype(np.uint8) << 7)).reshape(n, nb * 32)
        out[:, nb * 32:nb * 33] = code
    return out


def values(rec, dim, bits):
    """What records stand for, in 64 bits (NaN for a block of scale 255)."""
    n = rec.shape[0]
    nb = (dim + 31) // 32
    if bits == 4:
        q = rec[:, :nb * 16].reshape(n, nb, 16)
        q = np.stack((q & 15, q >> 4), 3).reshape(n, nb, 32)
        v = np.where(q & 8, -1.0, 1.0) * FP4[q & 7]
    else:
        q = rec[:, :nb * 32].reshape(n, nb, 32)
        v = np.where(q & 128, -1.0, 1.0) * np.append(FP8, np.nan)[q & 127]
    code = rec[:, nb * 4 * bits:nb * 4 * bits + nb]
    with np.errstate(invalid="ignore"):
        return (v * scale_of(code)[:, :, None]).reshape(n, nb * 32)[:, :dim]


def bf16(x):
    """x rounded to bf16 (nearest, ties to even), as fp32."""
    u = np.asarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32))


def mean(indptr, ids, rows):
    """Per destination: the mean of rows[ids[e]], and the mean of their magnitudes."""
    n, dim = len(indptr) - 1, rows.shape[1]
    out, mag = np.zeros((n, dim)), np.zeros((n, dim))
    for v in range(n):
        r = rows[ids[indptr[v]:indptr[v + 1]]]
        if len(r):
            out[v], mag[v] = r.mean(axis=0), np.abs(r).mean(axis=0)
    return out, mag


def distill(z, top, classes, labels, alpha, temperature):
    """(loss, gradient, scale of the loss's terms) row by row, in 64 bits."""
    z = np.asarray(z, np.float64)
    n, C = z.shape
    loss, size, grad = np.zeros(n), np.zeros(n), np.zeros((n, C))
    T = float(temperature)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for i in range(n):
            if np.all(z[i] == -np.inf):
                continue
            m = z[i].max()
            lq_t = (z[i] - m) / T - np.log(np.exp((z[i] - m) / T).sum())
            if alpha > 0:
                ok = [(c, float(t)) for c, t in zip(classes[i], top[i]) if 0 <= c < C and t != -np.inf]
                if ok:
                    t = np.array([x[1] for x in ok]) / T
                    lp = t - t.max() - np.log(np.exp(t - t.max()).sum())
                    p = np.exp(lp)
                    for (c, _), lpj, pj in zip(ok, lp, p):
                        if pj > 0 or np.isnan(pj):
                            loss[i] += alpha * T * T * pj * (lpj - lq_t[c])
                            size[i] += alpha * T * T * pj * (abs(lpj) + abs(lq_t[c]))
                        grad[i, c] -= alpha * T * pj / n
                    grad[i] += alpha * T * np.exp(lq_t) / n
            if labels is not None and alpha < 1 and 0 <= labels[i] < C:
                lq = z[i] - m - np.log(np.exp(z[i] - m).sum())
                loss[i] += (1 - alpha) * -lq[labels[i]]
                size[i] += (1 - alpha) * abs(lq[labels[i]])
                grad[i] += (1 - alpha) * np.exp(lq) / n
                grad[i, labels[i]] -= (1 - alpha) / n
    return loss, grad, size
