"""Plain definitions, in 64 bits, of dropout, the root-mean-square norm and the
cross-entropy over many classes (torch tensors, any device)."""
import numpy as np
import torch


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 (Salmon et al., SC'11) of arrays of counters: four arrays of words."""
    c = [np.asarray(v, np.uint64) & np.uint64(0xFFFFFFFF) for v in np.broadcast_arrays(c0, c1, c2, c3)]
    for r in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        a, b = np.uint64((k0 + r * 0x9E3779B9) & 0xFFFFFFFF), np.uint64((k1 + r * 0xBB67AE85) & 0xFFFFFFFF)
        low = np.uint64(0xFFFFFFFF)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ a, p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ b, p0 & low]
    return c


def threshold(p):
    return int(np.floor(65536.0 * float(np.float32(p)) + 0.5))


def keep(keys, dim, p, seed, layer=0, step=0):
    """Which elements of the rows with those keys are kept: bool [rows, dim]."""
    keys = np.asarray(keys).astype(np.int64)[:, None] & 0xFFFFFFFF
    o = np.arange(-(-dim // 8))[None, :]
    w = philox(keys, 0x80000000 + layer, o, step & 0xFFFFFFFF, seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=2)
    return torch.from_numpy(halves.reshape(keys.shape[0], -1)[:, :dim] >= threshold(p))


def drop(x, kept, p):
    """x (64 bits) dropped out: dropped elements 0 whatever they hold."""
    t = threshold(p)
    by = 0.0 if t >= 65536 else 65536.0 / (65536 - t)
    return torch.where(kept.to(x.device), x * by, torch.zeros_like(x))


def rms_norm(r, g, eps):
    return (r if g is None else g * r) / torch.sqrt(r.square().mean(1, keepdim=True) + eps)


def rms_norm_backward(dy, r, g, eps, carry=None):
    """(the gradient of r, that of the weight)"""
    s = 1 / torch.sqrt(r.square().mean(1, keepdim=True) + eps)
    a = dy if g is None else g * dy
    dr = s * (a - r * s * s * (a * r).mean(1, keepdim=True))
    return (dr if carry is None else dr + carry), (dy * r * s).sum(0)


def linear_loss(x, w, labels, bias=None):
    """(loss, dx, dw, dbias) of the mean cross-entropy; x and w in 64 bits."""
    n, classes = x.shape[0], w.shape[0]
    on = (labels >= 0) & (labels < classes)
    x = torch.where(on[:, None], x, torch.zeros_like(x))
    z = x @ w.t().contiguous()
    if bias is not None:
        z = z + bias
    top = z.max(1, keepdim=True)[0]
    on = on & (top[:, 0] > -np.inf)
    base = torch.where(top > -np.inf, top, torch.zeros_like(top))
    lse = (base + torch.exp(z - base).sum(1, keepdim=True).log())[:, 0]
    at = labels.clamp(0, classes - 1).long()[:, None]
    loss = torch.where(on, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse)).sum() / max(n, 1)
    g = torch.where(on[:, None], torch.exp(z - lse[:, None]), torch.zeros_like(z))
    g.scatter_add_(1, at, -on[:, None].to(g.dtype))
    return loss, g @ w / n, g.t().contiguous() @ x / n, g.sum(0) / n
