"""The operators of a vertex store and a model held in microscaled formats,
and the loss that trains such a model: measured through the package's entry
points (`own`), next to plain forms of the same operators.

A microscaled row is a record of bytes: the row's elements in blocks of 32,
each block a power-of-two scale (one byte, 2^(code - 127), 255 = not a
number) and 32 elements of 4 bits (sign, 0 .5 1 1.5 2 3 4 6) or of 8 bits
(e4m3).  First all blocks' elements (4 bits: the even element in the low
half of its byte), then the scales, then zeros up to a multiple of 16 bytes.
A block's scale is 2^(floor(log2(largest magnitude)) - 2) (8 bits: - 8), at
least 2^-127; elements are rounded to nearest, ties to even, and saturate.

A case is a dict of plain values.  `kind` says what one pass runs:
  write    rows into the store, by vertex id, and back out of it; with
           `turned`, a weight matrix [dim, n] whose columns become rows
  read     rows of the store by vertex id
  mean     the mean of every destination's sampled neighbours' rows
  linear   act(A W^T + A2 W2^T + b) of microscaled 4-bit rows and weights,
           A optionally by vertex id
  distill  the loss against a teacher's top logits and against labels, with
           its gradient in the logits
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16}
SIZE = {F32: 4, BF16: 2}


def listed():
    return [
        # a request of 64 vertices writes its 16 features into a small store
        {"name": "write_request", "kind": "write", "n": 64, "dim": 16, "bits": 8, "dtype": F32, "store": 10000, "turned": False},
        # the input vertices of a hub mini-batch written back in 4 bits
        {"name": "write_hubs", "kind": "write", "n": 350000, "dim": 128, "bits": 4, "dtype": BF16, "store": 2449029, "turned": False},
        # a few vertices of odd width read for one answer
        {"name": "read_request", "kind": "read", "n": 37, "dim": 75, "bits": 4, "dtype": BF16, "store": 100003},
        # the input rows of a product-graph mini-batch
        {"name": "read_products", "kind": "read", "n": 346000, "dim": 100, "bits": 4, "dtype": F32, "store": 2449029},
        # a request's own neighbourhood
        {"name": "mean_request", "kind": "mean", "n": 64, "fanout": 5, "dim": 16, "bits": 8, "dtype": F32, "store": 10000},
        # layer 0 of a product-graph mini-batch, straight from the store
        {"name": "mean_products", "kind": "mean", "n": 45000, "fanout": 15, "dim": 100, "bits": 4, "dtype": F32, "store": 2449029},
        # layer 0 of a hub mini-batch from an 8-bit store
        {"name": "mean_hubs", "kind": "mean", "n": 60000, "fanout": 25, "dim": 128, "bits": 8, "dtype": BF16, "store": 2449029},
        # one vertex through the last layer
        {"name": "linear_one", "kind": "linear", "n": 1, "d_in": 256, "d_out": 47, "two": True, "by_id": False, "relu": False, "dtype": F32, "store": 1},
        # layer 0 of a product-graph mini-batch, its own rows by id
        {"name": "linear_products", "kind": "linear", "n": 45000, "d_in": 100, "d_out": 256, "two": True, "by_id": True, "relu": True, "dtype": BF16, "store": 2449029},
        # a wide layer over many rows: bound by the products
        {"name": "linear_wide", "kind": "linear", "n": 8192, "d_in": 4096, "d_out": 4096, "two": False, "by_id": False, "relu": False, "dtype": BF16, "store": 8192},
        # a training batch's seeds, 47 classes, eight of the teacher's
        {"name": "distill_products", "kind": "distill", "n": 1000, "classes": 47, "top": 8, "dtype": F32, "alpha": 0.5, "temperature": 2.0, "labels": True},
        # many classes: one read and one write of a large logits array
        {"name": "distill_classes", "kind": "distill", "n": 4099, "classes": 32768, "top": 64, "dtype": BF16, "alpha": 0.75, "temperature": 1.5, "labels": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "read", "mean", "linear", "distill"])
    dtype = rng.choice([F32, BF16])
    if kind in ("write", "read"):
        c = {"kind": kind, "n": _log(rng, 1, 400000), "dim": _log(rng, 1, 1024), "bits": rng.choice([4, 8]), "dtype": dtype}
        c["n"] = min(c["n"], (1 << 26) // c["dim"])
        c["store"] = c["n"] + _log(rng, 1, 1000000)
        if kind == "write":
            c["turned"] = c["n"] <= 8192 and rng.random() < 0.4
        return c
    if kind == "mean":
        c = {"kind": kind, "n": _log(rng, 1, 60000), "fanout": _log(rng, 1, 40), "dim": _log(rng, 1, 512), "bits": rng.choice([4, 8]), "dtype": dtype}
        c["n"] = max(1, min(c["n"], (1 << 27) // (c["fanout"] * c["dim"])))
        c["store"] = _log(rng, 10, 2000000)
        return c
    if kind == "linear":
        c = {"kind": kind, "n": _log(rng, 1, 200000), "d_in": _log(rng, 1, 4096), "d_out": _log(rng, 1, 4096), "two": rng.random() < 0.5,
             "by_id": rng.random() < 0.5, "relu": rng.random() < 0.5, "dtype": dtype}
        c["n"] = max(1, min(c["n"], (1 << 36) // (c["d_in"] * c["d_out"]), (1 << 27) // c["d_out"], (1 << 27) // c["d_in"]))
        c["store"] = c["n"] + (_log(rng, 1, 100000) if c["by_id"] else 0)
        return c
    c = {"kind": kind, "classes": _log(rng, 2, 131072), "dtype": dtype, "alpha": rng.choice([0.0, 0.3, 0.9, 1.0]),
         "temperature": rng.choice([1.0, 1.0, 2.0, 4.0]), "labels": rng.random() < 0.7}
    c["n"] = max(1, min(_log(rng, 1, 60000), (1 << 26) // c["classes"]))
    c["top"] = min(c["classes"], _log(rng, 1, 256))
    return c


def record_bytes(dim, bits):
    blocks = (dim + 31) // 32
    return (blocks * 4 * bits + blocks + 15) // 16 * 16


# ---------------------------------------------------------------- plain form

def encode(x, bits):
    """The records of the rows of x."""
    n, dim = x.shape
    blocks = (dim + 31) // 32
    v = torch.zeros(n, blocks * 32, device=x.device)
    v[:, :dim] = x.float()
    v = v.view(n, blocks, 32)
    field = v.abs().amax(2).view(torch.int32) >> 23
    bad = field == 255
    code = (field - (2 if bits == 4 else 8)).clamp(min=0)
    v = v * ((254 - code) << 23).view(torch.float32)[:, :, None]
    v = torch.where(bad[:, :, None], torch.zeros_like(v), v)
    m = v.abs()
    if bits == 4:
        q = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5))
        q = q + 8 * torch.signbit(v)
        q = (q[:, :, 0::2] + 16 * q[:, :, 1::2]).view(n, blocks * 16)
    else:
        q = v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).reshape(n, blocks * 32)
    out = torch.zeros(n, record_bytes(dim, bits), dtype=torch.uint8, device=x.device)
    out[:, :blocks * 4 * bits] = q
    out[:, blocks * 4 * bits:blocks * 4 * bits + blocks] = torch.where(bad, 255, code).to(torch.uint8)
    return out


def decode(rec, dim, bits):
    """The rows that the records stand for, in fp32."""
    n = rec.shape[0]
    blocks = (dim + 31) // 32
    q = rec[:, :blocks * 4 * bits]
    code = rec[:, blocks * 4 * bits:blocks * 4 * bits + blocks].to(torch.int32)
    scale = torch.where(code == 0, 0x00400000, torch.where(code == 255, 0x7FC00000, code << 23)).view(torch.float32)
    if bits == 4:
        table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=rec.device)
        v = torch.stack((table[(q & 15).int()], table[(q >> 4).int()]), 2)
    else:
        v = q.contiguous().view(torch.float8_e4m3fn).float()
    return (v.reshape(n, blocks, 32) * scale[:, :, None]).reshape(n, blocks * 32)[:, :dim]


def _write(s):
    rec = encode(s["x"], s["bits"])
    if s["ids"] is None:
        return decode(rec, s["dim"], s["bits"]).to(s["x"].dtype)
    ids = s["ids"].long()
    s["store"][ids] = rec
    return decode(s["store"][ids], s["dim"], s["bits"]).to(s["x"].dtype)


def _read(s):
    return decode(s["store"][s["ids"].long()], s["dim"], s["bits"]).to(s["type"])


def _mean(s):
    indptr, rows = s["indptr"].long(), s["indices"].long()
    k = indptr[1:] - indptr[:-1]
    dst = torch.repeat_interleave(torch.arange(k.numel(), device=k.device), k, output_size=rows.numel())
    v = decode(s["store"][rows], s["dim"], s["bits"])
    total = torch.zeros(k.numel(), s["dim"], device=k.device).index_add_(0, dst, v)
    return (total / k.clamp(min=1)[:, None].float()).to(s["type"])


def _linear(s):
    a = s["a"] if s["ids"] is None else s["a"][s["ids"].long()]
    y = decode(a, s["d_in"], 4) @ decode(s["w"], s["d_in"], 4).t()
    if s["a2"] is not None:
        y = y + decode(s["a2"], s["d_in"], 4) @ decode(s["w2"], s["d_in"], 4).t()
    y = y + s["bias"]
    return (torch.where(y > 0, y, torch.zeros_like(y)) if s["relu"] else y).to(s["type"])


def _distill(s):
    z, n, t = s["logits"].float(), s["logits"].shape[0], s["temperature"]
    classes = z.shape[1]
    zt = z / t
    zt = zt - zt.amax(1, keepdim=True)
    logq = zt - zt.exp().sum(1, keepdim=True).log()
    ids = s["top_ids"].long()
    valid = (ids >= 0) & (ids < classes)
    any_valid = valid.any(1)
    at = ids.clamp(0, classes - 1)
    u = torch.where(valid, s["top"] / t, torch.full_like(s["top"], -math.inf))
    u = u - torch.where(any_valid, u.amax(1), torch.zeros_like(u[:, 0]))[:, None]
    e = u.exp()
    total = torch.where(any_valid, e.sum(1), torch.ones_like(e[:, 0]))[:, None]
    p = e / total
    kl = torch.where(p > 0, p * (u - total.log() - logq.gather(1, at)), torch.zeros_like(p)).sum(1)
    loss = s["alpha"] * t * t * kl
    grad = (s["alpha"] * t) * logq.exp() * any_valid[:, None].float()
    grad.scatter_add_(1, at, -(s["alpha"] * t) * p)
    if s["labels"] is not None:
        y = s["labels"].long()
        has = (y >= 0) & (y < classes)
        yc = y.clamp(0, classes - 1)[:, None]
        z1 = z - z.amax(1, keepdim=True)
        logq1 = z1 - z1.exp().sum(1, keepdim=True).log()
        weight = (1 - s["alpha"]) * has.float()
        loss = loss - weight * logq1.gather(1, yc)[:, 0]
        grad = grad + weight[:, None] * logq1.exp()
        grad.scatter_add_(1, yc, -weight[:, None])
    return {"loss": (loss.sum() / n).reshape(1), "grad": (grad / n).to(s["logits"].dtype)}


# ---------------------------------------------------------------- the framework's operators

def _own(s):
    import paper_2010_05337_amd as gmb
    kind = s["kind"]
    if kind == "write":
        if s["ids"] is None:
            rec = gmb.mx_quantise(s["x"], s["bits"])
            return gmb.mx_gather(None, rec, s["dim"], s["bits"], dtype=s["x"].dtype)
        gmb.mx_quantise(s["x"], s["bits"], ids=s["ids"], table=s["store"])
        return gmb.mx_gather(s["ids"], s["store"], s["dim"], s["bits"], dtype=s["x"].dtype)
    if kind == "read":
        return gmb.mx_gather(s["ids"], s["store"], s["dim"], s["bits"], dtype=s["type"])
    if kind == "mean":
        return gmb.mx_mean((s["indptr"], s["indices"]), s["store"], s["dim"], s["bits"], dtype=s["type"])
    if kind == "linear":
        return gmb.mx_linear(s["a"], s["w"], s["d_in"], bias=s["bias"], a2=s["a2"], w2=s["w2"], ids=s["ids"], relu=s["relu"], dtype=s["type"])
    loss, grad = gmb.distill_loss(s["logits"], s["top"], s["top_ids"], labels=s["labels"], alpha=s["alpha"], temperature=s["temperature"])
    return {"loss": loss, "grad": grad}


def run(state):
    if own:
        return _own(state)
    return {"write": _write, "read": _read, "mean": _mean, "linear": _linear, "distill": _distill}[state["kind"]](state)


# ---------------------------------------------------------------- inputs

def _features(n, dim, gen, dtype=torch.float32):
    """Rows of normal values whose widths differ from vertex to vertex."""
    x = torch.randn(n, dim, device="cuda", generator=gen)
    x *= torch.exp(0.7 * torch.randn(n, 1, device="cuda", generator=gen))
    return x.to(dtype)


def _store(rows, dim, bits, gen):
    """A store of `rows` records; made in pieces, a large one's fp32 rows are not held at once."""
    out = torch.empty(rows, record_bytes(dim, bits), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // max(dim, 32))
    for at in range(0, rows, step):
        end = min(rows, at + step)
        out[at:end] = encode(_features(end - at, dim, gen), bits)
    return out


def _distinct(n, rows, gen):
    """n different rows of `rows`, in no order."""
    if 4 * n > rows:
        return torch.randperm(rows, device="cuda", generator=gen)[:n].int()
    at = torch.randint(0, rows // n, (n,), device="cuda", generator=gen) + torch.arange(n, device="cuda") * (rows // n)
    return at[torch.randperm(n, device="cuda", generator=gen)].int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, n = case["kind"], case["n"]
    s = {"kind": kind}
    if kind == "write":
        s.update(dim=case["dim"], bits=case["bits"], ids=None)
        if case["turned"]:
            w = torch.randn(case["dim"], n, device="cuda", generator=gen) / math.sqrt(case["dim"])
            s["x"] = w.to(TYPES[case["dtype"]]).t()
        else:
            s["x"] = _features(n, case["dim"], gen, TYPES[case["dtype"]])
            s["store"] = torch.zeros(case["store"], record_bytes(case["dim"], case["bits"]), dtype=torch.uint8, device="cuda")
            s["ids"] = _distinct(n, case["store"], gen)
    elif kind == "read":
        s.update(dim=case["dim"], bits=case["bits"], type=TYPES[case["dtype"]])
        s["store"] = _store(case["store"], case["dim"], case["bits"], gen)
        s["ids"] = torch.randint(0, case["store"], (n,), device="cuda", generator=gen, dtype=torch.int32)
    elif kind == "mean":
        s.update(dim=case["dim"], bits=case["bits"], type=TYPES[case["dtype"]])
        s["store"] = _store(case["store"], case["dim"], case["bits"], gen)
        # most vertices have the whole fan-out, some fewer neighbours, some none
        u = torch.rand(n, device="cuda", generator=gen)
        k = torch.where(u < 0.7, torch.full_like(u, case["fanout"]), torch.floor((u - 0.7) / 0.3 * case["fanout"]))
        s["indptr"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        s["indptr"][1:] = torch.cumsum(k.long(), 0).int()
        s["indices"] = torch.randint(0, case["store"], (int(s["indptr"][-1]),), device="cuda", generator=gen, dtype=torch.int32)
    elif kind == "linear":
        d_in, d_out = case["d_in"], case["d_out"]
        s.update(d_in=d_in, relu=case["relu"], type=TYPES[case["dtype"]], a2=None, w2=None, ids=None)
        s["a"] = _store(case["store"], d_in, 4, gen)
        width = math.sqrt(6.0 / (d_in + d_out))
        s["w"] = encode((torch.rand(d_out, d_in, device="cuda", generator=gen) * 2 - 1) * width, 4)
        s["bias"] = torch.rand(d_out, device="cuda", generator=gen) * 0.2 - 0.1
        if case["by_id"]:
            s["ids"] = torch.randint(0, case["store"], (n,), device="cuda", generator=gen, dtype=torch.int32)
        if case["two"]:
            s["a2"] = _store(n, d_in, 4, gen)
            s["w2"] = encode((torch.rand(d_out, d_in, device="cuda", generator=gen) * 2 - 1) * width, 4)
    else:
        classes, top = case["classes"], case["top"]
        s.update(alpha=case["alpha"], temperature=case["temperature"], labels=None)
        s["logits"] = (torch.randn(n, classes, device="cuda", generator=gen) * 2).to(TYPES[case["dtype"]])
        step = torch.randint(1, classes // top + 1, (n, 1), device="cuda", generator=gen)
        start = torch.randint(0, classes, (n, 1), device="cuda", generator=gen)
        s["top_ids"] = ((start + step * torch.arange(top, device="cuda")) % classes).int()
        s["top"] = torch.sort(torch.randn(n, top, device="cuda", generator=gen) * 2 + 4, 1, descending=True)[0]
        # some vertices were given fewer of the teacher's logits, some none
        keep = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.9, top, torch.randint(0, top + 1, (n,), device="cuda", generator=gen))
        s["top_ids"][torch.arange(top, device="cuda") >= keep[:, None]] = -1
        if case["labels"]:
            y = torch.randint(0, classes, (n,), device="cuda", generator=gen, dtype=torch.int32)
            s["labels"] = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.8, y, -1).int()
    return s


def work(case):
    kind, n = case["kind"], case["n"]
    if kind == "distill":
        es = SIZE[case["dtype"]]
        cells = n * case["classes"]
        return {"bytes": 2 * es * cells + n * (8 * case["top"] + 4), "flops": 10 * cells}
    if kind == "linear":
        rec, pairs = record_bytes(case["d_in"], 4), 2 if case["two"] else 1
        read = pairs * (n + case["d_out"]) * rec + 4 * case["d_out"] + (4 * n if case["by_id"] else 0)
        return {"bytes": read + n * case["d_out"] * SIZE[case["dtype"]], "flops": 2 * pairs * n * case["d_in"] * case["d_out"]}
    rec, row = record_bytes(case["dim"], case["bits"]), case["dim"] * SIZE[case["dtype"]]
    if kind == "write":
        return {"bytes": n * (2 * row + rec + (0 if case["turned"] else 4)), "flops": 4 * n * case["dim"]}
    if kind == "read":
        return {"bytes": n * (row + rec + 4), "flops": n * case["dim"]}
    edges = n * case["fanout"] * 0.85
    rows = case["store"] * -math.expm1(-edges / case["store"])
    return {"bytes": rows * rec + 4 * edges + 4 * n + n * row, "flops": edges * case["dim"]}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _values(rec, dim, bits):
    """What records stand for, from the formats' fields."""
    blocks = (dim + 31) // 32
    raw = rec[:, :blocks * 4 * bits].double()
    if bits == 4:
        high = torch.floor(raw / 16)
        raw = torch.stack((raw - 16 * high, high), 2).reshape(rec.shape[0], blocks * 32)
    half = 8.0 if bits == 4 else 128.0
    sign = 1 - 2 * (raw >= half).double()
    mag = torch.remainder(raw, half)
    per = 2.0 if bits == 4 else 8.0             # mantissa steps of an exponent
    e, m = torch.floor(mag / per), torch.remainder(mag, per) / per
    bias = 1.0 if bits == 4 else 7.0
    v = sign * torch.where(e > 0, (1 + m) * torch.exp2(e - bias), m * 2.0 ** (1 - bias))
    scale = rec[:, blocks * 4 * bits:blocks * 4 * bits + blocks].double()
    scale = torch.where(scale == 255, torch.full_like(scale, math.nan), torch.exp2(scale - 127))
    return (v.view(-1, blocks, 32) * scale[:, :, None]).reshape(-1, blocks * 32)[:, :dim]


def _rounded(x, bits):
    """x as a microscaled format holds it: the nearest of the format's values at the block's scale."""
    n, dim = x.shape
    blocks = (dim + 31) // 32
    v = torch.nn.functional.pad(x.double(), (0, blocks * 32 - dim)).view(n, blocks, 32)
    big = v.abs().amax(2, keepdim=True)
    exponent = torch.where(big > 0, torch.frexp(big)[1].double() - 1, -200.0 * torch.ones_like(big))
    top = 2.0 if bits == 4 else 8.0
    scale = torch.exp2((exponent - top).clamp(min=-127.0))
    m = v.abs() / scale
    lowest, digits, most = (0.0, 1.0, 6.0) if bits == 4 else (-6.0, 3.0, 448.0)
    unit = torch.exp2((torch.frexp(m)[1].double() - 1).clamp(min=lowest) - digits)
    r = (torch.round(m / unit) * unit).clamp(max=most)      # round() takes ties to even
    out = torch.where(v < 0, -r, r) * scale
    return out.reshape(n, blocks * 32)[:, :dim]


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "write":
        return _rounded(s["x"], s["bits"])
    if kind == "read":
        return _values(s["store"][s["ids"].long()], s["dim"], s["bits"])
    if kind == "mean":
        ptr = s["indptr"].tolist()
        k = torch.tensor([b - a for a, b in zip(ptr, ptr[1:])], device="cuda")
        out = torch.zeros(k.numel(), s["dim"], dtype=torch.float64, device="cuda")
        start = s["indptr"][:-1].long()
        for j in range(int(k.max())):                       # the j-th neighbour of all that have one
            has = torch.nonzero(k > j)[:, 0]
            out[has] += _values(s["store"][s["indices"][start[has] + j].long()], s["dim"], s["bits"])
        return out / k.clamp(min=1)[:, None]
    if kind == "linear":
        a = s["a"] if s["ids"] is None else s["a"].index_select(0, s["ids"].long())
        y = torch.addmm(s["bias"].double(), _values(a, s["d_in"], 4), _values(s["w"], s["d_in"], 4).t().contiguous())
        if s["a2"] is not None:
            y.addmm_(_values(s["a2"], s["d_in"], 4), _values(s["w2"], s["d_in"], 4).t().contiguous())
        return y.clamp(min=0) if s["relu"] else y
    z, t, alpha = s["logits"].double(), s["temperature"], s["alpha"]
    n, classes = z.shape
    lse = torch.logsumexp(z / t, 1)
    grad = torch.zeros_like(z)
    valid = s["top_ids"] >= 0
    ids = torch.where(valid, s["top_ids"], 0).long()
    p = torch.softmax(torch.where(valid, s["top"].double() / t, -math.inf), 1).nan_to_num(0.0)
    has = valid.any(1)
    terms = torch.xlogy(p, p) - p * (z.gather(1, ids) / t - lse[:, None])
    loss = alpha * t * t * terms.sum(1)
    grad = alpha * t * has[:, None] * torch.exp(z / t - lse[:, None])
    grad.scatter_add_(1, ids, -alpha * t * p)
    if s["labels"] is not None:
        rows = torch.nonzero(s["labels"] >= 0)[:, 0]
        y = s["labels"][rows].long()
        lse1 = torch.logsumexp(z[rows], 1)
        loss[rows] += (1 - alpha) * (lse1 - z[rows, y])
        grad[rows] += (1 - alpha) * torch.exp(z[rows] - lse1[:, None])
        grad[rows, y] -= 1 - alpha
    return {"loss": (loss.sum() / n).reshape(1), "grad": grad / n}
