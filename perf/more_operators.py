"""Dropout from a counter-based generator, the root-mean-square norm with the
residual's addition, and the cross-entropy over many classes without logits:
measured through the package's entry points (`own`), next to plain forms of
the same operators.

A case is a dict of plain values.  `kind` says what one pass runs:
  dropout    [residual +] x with elements dropped and the others scaled
  norm       r = residual + x (x dropped out first, if p > 0) and its norm
             y = g r / sqrt(mean(r^2) + eps); with `bits`, y in microscaled
             records, read back as the values they stand for
  norm_back  the gradients of x, of the residual and of g from those of y
             and (with `carry`) of r
  loss       the mean over the rows of -log softmax(x W^T + b)[label], with
             `grad` its gradients in x, W and b; with `turned` W is given as
             a [d, classes] matrix

Which elements are dropped: Philox4x32-10 (Salmon et al., SC'11) keyed by the
seed's two words, counter (row's key, 2^31 + layer, column / 8, step); the
columns 8 c .. 8 c + 7 take the low and high halves of its words in order, and
an element is dropped where its 16 bits are below round(65536 p).  Kept ones
are scaled by 65536 / (65536 - round(65536 p)).
"""
import math

import numpy as np
import torch

own = False

F32, BF16 = "f32", "bf16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16}
SIZE = {F32: 4, BF16: 2}
EPS = 1e-6


def listed():
    return [
        # the hidden rows of a small request's 64 seeds
        {"name": "dropout_request", "kind": "dropout", "n": 64, "dim": 16, "dtype": F32, "p": 0.5, "layer": 1, "ids": True, "residual": False},
        # the hidden rows of a product-graph mini-batch, the same vertex the same mask
        {"name": "dropout_products", "kind": "dropout", "n": 45000, "dim": 256, "dtype": F32, "p": 0.5, "layer": 0, "ids": True, "residual": False},
        # the input rows of a hub mini-batch, on top of a residual
        {"name": "dropout_hubs", "kind": "dropout", "n": 350000, "dim": 128, "dtype": BF16, "p": 0.1, "layer": 3, "ids": False, "residual": True},
        # one vertex served: the sum and its norm as an 8-bit record
        {"name": "norm_one", "kind": "norm", "n": 1, "dim": 256, "dtype": BF16, "p": 0.0, "residual": True, "bits": 8},
        # a training step's hidden rows, with dropout and residual
        {"name": "norm_products", "kind": "norm", "n": 45000, "dim": 256, "dtype": F32, "p": 0.5, "residual": True, "bits": 0},
        # wide rows into the 8-bit store
        {"name": "norm_wide", "kind": "norm", "n": 8192, "dim": 4096, "dtype": BF16, "p": 0.0, "residual": True, "bits": 8},
        # the backward of the training step's hidden rows
        {"name": "norm_back_products", "kind": "norm_back", "n": 45000, "dim": 256, "dtype": F32, "p": 0.5, "carry": True},
        # the backward of wide rows
        {"name": "norm_back_wide", "kind": "norm_back", "n": 8192, "dim": 4096, "dtype": BF16, "p": 0.0, "carry": True},
        # a training batch's seeds against 47 classes
        {"name": "loss_products", "kind": "loss", "n": 1000, "d": 256, "classes": 47, "dtype": F32, "bias": True, "grad": True, "turned": True},
        # every vertex of a 100,000-vertex graph a class, the embedding table the weights
        {"name": "loss_vertices", "kind": "loss", "n": 4000, "d": 256, "classes": 100000, "dtype": BF16, "bias": False, "grad": True, "turned": False},
        # the same kind of head in fp32, over a smaller table
        {"name": "loss_vertices_f32", "kind": "loss", "n": 4000, "d": 256, "classes": 20011, "dtype": F32, "bias": True, "grad": True, "turned": False},
        # a wide head: bound by the products
        {"name": "loss_wide", "kind": "loss", "n": 8192, "d": 1024, "classes": 32768, "dtype": BF16, "bias": False, "grad": True, "turned": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["dropout", "norm", "norm_back", "loss", "loss"])
    dtype = rng.choice([F32, BF16])
    p = rng.choice([0.1, 0.25, 0.5, 0.9])
    if kind == "loss":
        c = {"kind": kind, "n": _log(rng, 1, 16384), "d": _log(rng, 1, 2048), "classes": _log(rng, 2, 200000), "dtype": dtype,
             "bias": rng.random() < 0.5, "grad": rng.random() < 0.8}
        c["d"] = max(1, min(c["d"], (1 << 25) // c["classes"]))
        c["n"] = max(1, min(c["n"], (1 << 28) // c["classes"], (1 << (38 if dtype == BF16 else 36)) // (c["classes"] * c["d"])))
        c["turned"] = rng.random() < 0.3
        return c
    c = {"kind": kind, "n": _log(rng, 1, 350000), "dim": _log(rng, 1, 16384), "dtype": dtype}
    c["n"] = max(1, min(c["n"], (1 << 25) // c["dim"]))
    if kind == "dropout":
        c.update(p=p, layer=rng.randrange(8), ids=rng.random() < 0.5, residual=rng.random() < 0.5)
    elif kind == "norm":
        c.update(p=p if rng.random() < 0.5 else 0.0, residual=rng.random() < 0.7, bits=rng.choice([0, 0, 4, 8]))
    else:
        c.update(p=p if rng.random() < 0.5 else 0.0, carry=rng.random() < 0.7)
    return c


# ---------------------------------------------------------------- plain form

def _threshold(p):
    return int(math.floor(65536 * p + 0.5))


def _scale(p):
    return 65536.0 / (65536 - _threshold(p))


def kept(key, dim, p, seed, layer):
    """Which elements of the rows with those keys are kept."""
    low = 0xFFFFFFFF
    blocks = (dim + 7) // 8
    c = [key.long()[:, None].expand(-1, blocks), torch.full((1, 1), (1 << 31) + layer, device=key.device),
         torch.arange(blocks, device=key.device)[None, :], torch.zeros((1, 1), dtype=torch.long, device=key.device)]
    k0, k1 = seed & low, (seed >> 32) & low

    def turn(c, r):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        return [((b >> 32) & low) ^ c[1] ^ ((k0 + r * 0x9E3779B9) & low), b & low,
                ((a >> 32) & low) ^ c[3] ^ ((k1 + r * 0xBB67AE85) & low), a & low]

    c = turn(turn(turn(turn(turn(c, 0), 1), 2), 3), 4)
    c = turn(turn(turn(turn(turn(c, 5), 6), 7), 8), 9)
    words = torch.stack([w.expand(key.numel(), blocks) for w in c], 2)
    halves = torch.stack((words & 0xFFFF, words >> 16), 3).reshape(key.numel(), blocks * 8)
    return halves[:, :dim] >= _threshold(p)


def _dropped(x, s):
    x = x.float()
    if s["p"] == 0:
        return x
    key = s["ids"] if s.get("ids") is not None else torch.arange(x.shape[0], device=x.device)
    return torch.where(kept(key, x.shape[1], s["p"], s["seed"], s["layer"]), x * _scale(s["p"]), torch.zeros_like(x))


def _dropout(s):
    y = _dropped(s["x"], s)
    return (y if s["residual"] is None else s["residual"].float() + y).to(s["x"].dtype)


def _microscaled(x, bits):
    """The values that microscaled blocks of 32 elements hold for the rows of x."""
    n, dim = x.shape
    blocks = (dim + 31) // 32
    v = torch.zeros(n, blocks * 32, device=x.device)
    v[:, :dim] = x
    v = v.view(n, blocks, 32)
    code = ((v.abs().amax(2).view(torch.int32) >> 23) - (2 if bits == 4 else 8)).clamp(min=1)
    up, down = (code << 23).view(torch.float32)[:, :, None], ((254 - code) << 23).view(torch.float32)[:, :, None]
    v = v * down
    if bits == 4:
        m = v.abs()
        q = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5))
        q = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=x.device)[q]
        v = torch.where(v < 0, -q, q)
    else:
        v = v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()
    return (v * up).reshape(n, blocks * 32)[:, :dim]


def _norm(s):
    r = _dropped(s["x"], s)
    if s["residual"] is not None:
        r = s["residual"].float() + r
    r = r.to(s["x"].dtype)
    v = r.float()
    y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["g"]
    if s["bits"]:
        return {"y": _microscaled(y, s["bits"]).to(torch.bfloat16), "r": r}
    return {"y": y.to(s["x"].dtype), "r": r}


def _norm_back(s):
    v, dy = s["r"].float(), s["dy"].float()
    inv = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    xhat, gy = v * inv, dy * s["g"]
    dr = inv * (gy - xhat * (gy * xhat).mean(1, keepdim=True))
    if s["carry"] is not None:
        dr = s["carry"].float() + dr
    out = {"residual": dr.to(s["r"].dtype), "g": (dy * xhat).sum(0)}
    if s["p"]:
        out["x"] = _dropped(dr, s).to(s["r"].dtype)
    return out


def _loss(s):
    x, w = s["x"].float(), s["w"].float()
    n = x.shape[0]
    z = x @ (w if s["turned"] else w.t())
    classes = z.shape[1]
    if s["bias"] is not None:
        z = z + s["bias"]
    y = s["labels"].long()
    has = ((y >= 0) & (y < classes)).float()
    at = y.clamp(0, classes - 1)[:, None]
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    total = e.sum(1, keepdim=True)
    loss = ((has * (total.log() - z.gather(1, at))[:, 0]).double().sum() / n).float().reshape(1)
    if not s["grad"]:
        return {"loss": loss}
    g = e / total
    g.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    g = g * (has / n)[:, None]
    out = {"loss": loss, "x": (g @ (w.t() if s["turned"] else w)).to(s["x"].dtype),
           "w": (x.t() @ g if s["turned"] else g.t() @ x).to(s["w"].dtype)}
    if s["bias"] is not None:
        out["b"] = g.sum(0)
    return out


# ---------------------------------------------------------------- the framework's operators

def _own(s):
    import paper_2010_05337_amd as gmb
    kind = s["kind"]
    if kind == "loss":
        w = s["w"].t() if s["turned"] else s["w"]
        loss, grads = gmb.linear_loss(s["x"], w, s["labels"], bias=s["bias"], grad=s["grad"])
        if not s["grad"]:
            return {"loss": loss}
        out = {"loss": loss, "x": grads.x, "w": grads.w.t() if s["turned"] else grads.w}
        if s["bias"] is not None:
            out["b"] = grads.bias
        return out
    drop = gmb.Dropout(s["p"], s["seed"], layer=s["layer"]) if s["p"] else None
    if kind == "dropout":
        return gmb.dropout(s["x"], drop, ids=s["ids"], residual=s["residual"])
    if kind == "norm":
        y, r = gmb.rms_norm(s["x"], s["g"], EPS, residual=s["residual"], dropout=drop, bits=s["bits"] or None)
        if s["bits"]:
            y = gmb.mx_gather(None, y, s["x"].shape[1], s["bits"], dtype=torch.bfloat16)
        return {"y": y, "r": r}
    grads = gmb.rms_norm_backward(s["dy"], s["r"], s["g"], EPS, carry=s["carry"], dropout=drop)
    out = {"residual": grads.residual, "g": grads.weight}
    if s["p"]:
        out["x"] = grads.x
    return out


def run(state):
    if own:
        return _own(state)
    return {"dropout": _dropout, "norm": _norm, "norm_back": _norm_back, "loss": _loss}[state["kind"]](state)


# ---------------------------------------------------------------- inputs

def _rows(n, dim, gen, dtype):
    """Rows of normal values whose widths differ from vertex to vertex."""
    x = torch.randn(n, dim, device="cuda", generator=gen)
    x *= torch.exp(0.7 * torch.randn(n, 1, device="cuda", generator=gen))
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, n, dtype = case["kind"], case["n"], TYPES[case["dtype"]]
    s = {"kind": kind}
    if kind == "loss":
        d, classes = case["d"], case["classes"]
        w = torch.randn(classes, d, device="cuda", generator=gen) * (2 / math.sqrt(d))
        y = torch.randint(0, classes, (n,), device="cuda", generator=gen, dtype=torch.int32)
        # rows that lean towards their label's weights, some by far, some not at all
        lean = torch.rand(n, 1, device="cuda", generator=gen) * 0.6
        x = torch.randn(n, d, device="cuda", generator=gen) + lean * (math.sqrt(d) / 2) * w[y.long()]
        y = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.9, y, -1).int()
        s.update(x=x.to(dtype), labels=y, turned=case["turned"], grad=case["grad"], bias=None)
        s["w"] = (w.t().contiguous() if case["turned"] else w).to(dtype)
        if case["bias"]:
            s["bias"] = torch.randn(classes, device="cuda", generator=gen) * 0.1
        return s
    dim = case["dim"]
    s.update(p=case["p"], seed=(seed * 0x9E3779B97F4A7C15 + 12345) & 0x7FFFFFFFFFFFFFFF, layer=case.get("layer", 0), ids=None)
    if kind == "dropout":
        s["x"] = _rows(n, dim, gen, dtype)
        s["residual"] = _rows(n, dim, gen, dtype) if case["residual"] else None
        if case["ids"]:
            s["ids"] = torch.randint(0, 2449029, (n,), device="cuda", generator=gen, dtype=torch.int32)
        return s
    s["g"] = 1 + 0.2 * torch.randn(dim, device="cuda", generator=gen)
    if kind == "norm":
        s.update(x=_rows(n, dim, gen, dtype), bits=case["bits"], residual=_rows(n, dim, gen, dtype) if case["residual"] else None)
        return s
    s.update(r=_rows(n, dim, gen, dtype), dy=(torch.randn(n, dim, device="cuda", generator=gen) * 0.1).to(dtype), carry=None)
    if case["carry"]:
        s["carry"] = (torch.randn(n, dim, device="cuda", generator=gen) * 0.1).to(dtype)
    return s


def work(case):
    n, es = case["n"], SIZE[case["dtype"]]
    if case["kind"] == "loss":
        d, classes, products = case["d"], case["classes"], 3 if case["grad"] else 1
        sides = (n + classes) * d * es * (2 if case["grad"] else 1)
        bias = 4 * classes * ((1 if case["bias"] else 0) + (1 if case["bias"] and case["grad"] else 0))
        return {"bytes": sides + 4 * n + bias, "flops": 2 * products * n * d * classes + 4 * n * classes}
    cells = n * case["dim"]
    draws = 8 * cells if case["p"] else 0         # ten rounds of six operations for eight elements
    if case["kind"] == "dropout":
        return {"bytes": es * cells * (3 if case["residual"] else 2) + (4 * n if case["ids"] else 0), "flops": draws}
    if case["kind"] == "norm":
        y = {0: es, 4: 17 / 32, 8: 33 / 32}[case["bits"]]
        back = 0 if not case["bits"] else y + 2   # records are read back as bf16
        sums = es if case["residual"] or case["p"] else 0   # (the sum of x alone is x)
        return {"bytes": cells * (es + (es if case["residual"] else 0) + sums + y + back) + 4 * case["dim"], "flops": draws + 5 * cells}
    return {"bytes": cells * es * (3 + (1 if case["carry"] else 0) + (1 if case["p"] else 0)) + 8 * case["dim"], "flops": draws + 10 * cells}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _mask(key, dim, p, seed, layer):
    """Which elements are kept, from the generator's definition in unsigned words on the host."""
    word = np.uint64(0xFFFFFFFF)
    blocks = -(-dim // 8)
    a = np.repeat(key.astype(np.uint64), blocks)
    b = np.full(a.size, 0x80000000 + layer, np.uint64)
    c = np.tile(np.arange(blocks, dtype=np.uint64), key.size)
    d = np.zeros(a.size, np.uint64)
    k0, k1 = seed % (1 << 32), seed >> 32
    for _ in range(10):
        x, y = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = (y >> np.uint64(32)) ^ b ^ np.uint64(k0), y & word, (x >> np.uint64(32)) ^ d ^ np.uint64(k1), x & word
        k0, k1 = (k0 + 0x9E3779B9) % (1 << 32), (k1 + 0xBB67AE85) % (1 << 32)
    halves = np.empty((a.size, 8), np.uint32)
    for i, w in enumerate((a, b, c, d)):
        halves[:, 2 * i], halves[:, 2 * i + 1] = w & np.uint64(0xFFFF), w >> np.uint64(16)
    return torch.from_numpy(halves.reshape(key.size, blocks * 8)[:, :dim] >= int(round(p * 65536))).cuda()


def _rounded(x, bits):
    """x as a microscaled format holds it: the nearest of the format's values at the block's scale."""
    n, dim = x.shape
    blocks = (dim + 31) // 32
    v = torch.nn.functional.pad(x, (0, blocks * 32 - dim)).view(n, blocks, 32)
    big = v.abs().amax(2, keepdim=True)
    exponent = torch.where(big > 0, torch.frexp(big)[1].double() - 1, -100.0 * torch.ones_like(big))
    scale = torch.exp2(exponent - (2.0 if bits == 4 else 8.0))
    m = v.abs() / scale
    lowest, digits, most = (0.0, 1.0, 6.0) if bits == 4 else (-6.0, 3.0, 448.0)
    unit = torch.exp2((torch.frexp(m)[1].double() - 1).clamp(min=lowest) - digits)
    r = (torch.round(m / unit) * unit).clamp(max=most)      # round() takes ties to even
    return (torch.where(v < 0, -r, r) * scale).reshape(n, blocks * 32)[:, :dim]


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "loss":
        x, w = s["x"].double(), s["w"].double()
        w = w.t() if s["turned"] else w
        z = torch.matmul(x, w.t())
        if s["bias"] is not None:
            z += s["bias"].double()
        rows = torch.nonzero(s["labels"] >= 0)[:, 0]
        y = s["labels"][rows].long()
        lse = torch.logsumexp(z, 1)
        n = x.shape[0]
        loss = ((lse[rows] - z[rows, y]).sum() / n).reshape(1)
        if not s["grad"]:
            return {"loss": loss}
        g = z.sub_(lse[:, None]).exp_()
        g[rows, y] -= 1
        g[s["labels"] < 0] = 0
        g /= n
        dw = torch.matmul(g.t(), x)
        out = {"loss": loss, "x": torch.matmul(g, w), "w": dw.t().contiguous() if s["turned"] else dw}
        if s["bias"] is not None:
            out["b"] = g.sum(0)
        return out
    dtype = (s["x"] if "x" in s else s["r"]).dtype

    def dropped(v):
        if not s["p"]:
            return v
        key = np.arange(v.shape[0]) if s["ids"] is None else s["ids"].cpu().numpy()
        keep = _mask(key, v.shape[1], s["p"], s["seed"], s["layer"])
        return torch.where(keep, v / (1 - round(s["p"] * 65536) / 65536), 0.0)

    if kind == "dropout":
        y = dropped(s["x"].double())
        return y if s["residual"] is None else y + s["residual"].double()
    g = s["g"].double()
    if kind == "norm":
        r = dropped(s["x"].double())
        if s["residual"] is not None:
            r = r + s["residual"].double()
        held = r.to(dtype).double()                          # y is the norm of r as it is stored
        y = g * held / torch.sqrt(held.square().mean(1, keepdim=True) + EPS)
        return {"y": _rounded(y, s["bits"]) if s["bits"] else y, "r": r}
    r, dy = s["r"].double(), s["dy"].double()
    size = torch.sqrt(r.square().mean(1, keepdim=True) + EPS)
    along = (g * dy * r).mean(1, keepdim=True)
    dr = g * dy / size - r * along / size ** 3
    if s["carry"] is not None:
        dr = dr + s["carry"].double()
    out = {"residual": dr, "g": (dy * r / size).sum(0)}
    if s["p"]:
        out["x"] = dropped(dr)
    return out
