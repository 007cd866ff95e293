"""The cross-entropy over many classes on the GPU against its definition in 64
bits.

Bounds.  A logit is a sum of d products: in bf16 they are exact, in fp32 an
operand's two parts lose below 2^-22 of it and 2^-38 of the largest, the fourth
part product below 2^-22; the sum rounds at every addition at most, U = 2^-24 of
the terms' magnitudes (three chains in fp32), its scale and bias once more.
With dz that error, a softmax is off by 2 dz (its own logit and the others') and
its exponentials' arguments, sums and quotient: an argument down to -32 keeps 2
x 32 + 4 half-steps, sums of positive terms add one a link of their chains (64
registers, exchanges, tiles an eighth apart): REL = 400 U covers them for up to
100 tiles an eighth.  Its gradient is then rounded to bf16 (2^-8) or cut in two
(2^-22 and 2^-38), and the products add as above.  A result below 2^-126 is one
of the multiples of 2^-149: half of that, for each of its two factors."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import head_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402

U, ULOW = 2.0 ** -24, 2.0 ** -8
TINY = 2.0 ** -149
REL = 400 * U
TYPES = [torch.float32, torch.bfloat16]


def problem(n, d, classes, dtype, seed, bias=True, none=0.2):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(classes, d, device="cuda", generator=gen) * (2 / math.sqrt(d))
    y = torch.randint(0, classes, (n,), device="cuda", generator=gen, dtype=torch.int32)
    lean = torch.rand(n, 1, device="cuda", generator=gen) * 0.6
    x = torch.randn(n, d, device="cuda", generator=gen) + lean * (math.sqrt(d) / 2) * w[y.long()]
    b = torch.randn(classes, device="cuda", generator=gen) if bias else None
    y = torch.where(torch.rand(n, device="cuda", generator=gen) < 1 - none, y, -1).int()
    return x.to(dtype), w.to(dtype), y, b


def near(got, want, tol, what):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((got - want).abs()[bad].max()), float(tol[bad].min()) if tol.dim() else float(tol),
                           bad.nonzero()[:3].tolist())


def check(x, w, y, b, got, grads):
    """Against the definition, with the bounds above (all on the GPU in 64 bits)."""
    low = x.dtype is torch.bfloat16
    n, d = x.shape
    classes = w.shape[0]
    on = (y >= 0) & (y < classes)
    X = torch.where(on[:, None], x.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    W, B = w.double(), None if b is None else b.double()
    loss, dx, dw, db = head_ref.linear_loss(X, W, y, B)
    ax, aw = X.abs(), W.abs()
    part = (lambda v, top: torch.zeros_like(v)) if low else (lambda v, top: 2.0 ** -22 * v + 2.0 ** -38 * top)
    ex, ew = part(ax, ax.amax(1, keepdim=True) if n else 0.0), part(aw, aw.max())
    chain = (d + 4 if low else 3 * d + 8) * U + (0.0 if low else 2.0 ** -22)
    dz = ax @ ew.t() + (ex @ aw.t()) + chain * (ax @ aw.t())
    if b is not None:
        dz = dz + 2 * U * (ax @ aw.t() + torch.where(b.isinf(), 0.0, b.abs()).double())
    worst = dz.amax(1)
    terms = (2 * worst + REL * 1.0 + 40 * U)[on]
    near(got, loss.reshape(1), (terms.sum() / max(n, 1) + 4 * U * loss.abs()).reshape(1) * 1.01, "loss")
    if not grads:
        return
    z = X @ W.t().contiguous() + (0 if B is None else B)
    p = torch.where(on[:, None], torch.softmax(z, 1), torch.zeros((), dtype=torch.float64, device="cuda"))
    g = p.clone()
    g[on, y[on].long()] -= 1
    # (the bound on arguments below -32: e^-32 of the row's sum)
    eg = p * (dz + worst[:, None] + REL) * 1.01 + 1e-13 * on[:, None]
    eg_sum = eg + U * g.abs()
    eg = eg + (ULOW * g.abs() if low else 2.0 ** -22 * g.abs() + 2.0 ** -38) * on[:, None]
    ag = g.abs() + eg
    if grads.x is not None:
        sums = (classes + 8) * (1 if low else 3) * U + (0.0 if low else 2.0 ** -22)
        # (a chain of classes: its links' errors are bounded by a random walk's eight deviations)
        sums = min(sums, 8 * math.sqrt(classes + 8) * 2 * U + (0.0 if low else 2.0 ** -22) + 64 * U)
        tol = (eg @ aw + ag @ ew + sums * (ag @ aw)) / n + 4 * U * dx.abs()
        near(grads.x, dx, tol * 1.01 + TINY + (ULOW * (dx.abs() + tol) if low else 0), "dx")
    if grads.w is not None:
        xt = part(ax, ax.max())
        sums = (n + 8) * (1 if low else 3) * U + (0.0 if low else 2.0 ** -22)
        sums = min(sums, 8 * math.sqrt(n + 8) * 2 * U + (0.0 if low else 2.0 ** -22) + 64 * U)
        tol = (eg.t() @ ax + ag.t() @ xt + sums * (ag.t() @ ax)) / n + 4 * U * dw.abs()
        near(grads.w, dw, tol * 1.01 + TINY + (ULOW * (dw.abs() + tol) if low else 0), "dw")
    if grads.bias is not None:
        near(grads.bias, db, (eg_sum.sum(0) + (n + 8) * U * g.abs().sum(0)) / n * 1.01 + 2 * U * db.abs(), "dbias")


# a head that fits LDS, one in small tiles, one in large ones
HEADS = [(60, 40, 200), (60, 140, 1000), (2100, 64, 5000)]
# rows, columns and classes around tiles (64, 256), stages (32, 64) and their padding
SIZES = [(1, 1, 1), (1, 5, 2), (3, 16, 8), (64, 16, 47), (5, 64, 127), (127, 33, 128), (128, 100, 129), (129, 128, 256), (200, 63, 257),
         (300, 65, 47), (1000, 256, 47), (257, 300, 1000), (1, 256, 5000), (40, 129, 5003), (513, 7, 640), (31, 700, 300),
         (1500, 48, 172), (2, 2048, 33), (4096, 16, 40), (4097, 16, 40), (50, 1024, 16), (50, 1025, 16), (33, 64, 256),
         (33, 64, 257), (2048, 96, 5000)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_loss_and_gradients(size, dtype):
    for bias in (True, False):
        x, w, y, b = problem(*size, dtype, 1, bias)
        loss, grads = gmb.linear_loss(x, w, y, bias=b)
        assert grads.x.dtype is dtype and grads.w.dtype is dtype and (grads.bias is None) == (not bias)
        check(x, w, y, b, loss, grads)
        alone, none = gmb.linear_loss(x, w, y, bias=b, grad=False)
        assert torch.equal(alone, loss) and none == (None, None, None)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 5, 2), (129, 100, 47), (300, 64, 300), (64, 256, 1000), (700, 20, 130)], ids=str)
def test_layouts_and_strides(size, dtype):
    n, d, classes = size
    x, w, y, b = problem(*size, dtype, 2)
    loss, grads = gmb.linear_loss(x, w, y, bias=b)
    # a [d, classes] matrix: its gradient has its layout
    m = w.t().contiguous()
    loss2, g2 = gmb.linear_loss(x, m.t(), y, bias=b)
    assert torch.equal(loss2, loss) and torch.equal(g2.x, grads.x) and torch.equal(g2.bias, grads.bias)
    check(x, w, y, b, loss2, g2)
    if d > 1 and classes > 1:
        assert g2.w.t().is_contiguous()
    # rows at strides, nothing contiguous, an address off 16 bytes
    xs = torch.full((n, d + 3), 9.0, device="cuda").to(dtype)
    xs[:, :d] = x
    ws = torch.full((classes, 2 * d + 5), 9.0, device="cuda").to(dtype)
    ws[:, 1:2 * d + 1:2] = w
    for xx, ww in [(xs[:, :d], w), (x, ws[:, 1:2 * d + 1:2])]:
        loss3, g3 = gmb.linear_loss(xx, ww, y, bias=b)
        assert torch.equal(loss3, loss) and torch.equal(g3.x, grads.x) and torch.equal(g3.w, grads.w)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 65536, 3), (3, 20_000, 700), (40, 60_000, 300), (300, 5000, 1), (17, 9, 4000), (70, 1025, 4100),
                                  (100_000, 3, 2)], ids=str)
def test_long_rows_and_lean_heads(size, dtype):
    x, w, y, b = problem(*size, dtype, 17)
    loss, grads = gmb.linear_loss(x, w, y, bias=b)
    check(x, w, y, b, loss, grads)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", [(40, 64, 30), (300, 128, 700)], ids=str)
def test_weights_that_are_broadcast(size, dtype):
    """Strides of zero: every element has a gradient of its own."""
    n, d, classes = size
    x, w, y, b = problem(*size, dtype, 18)
    for wide in (w[0].expand(classes, d), w[:, :1].expand(classes, d), w[0, 0].expand(classes, d)):
        loss, g = gmb.linear_loss(x, wide, y, bias=b)
        check(x, wide, y, b, loss, g)
        dense, h = gmb.linear_loss(x, wide.contiguous(), y, bias=b)
        assert torch.equal(loss, dense) and all(torch.equal(p, q) for p, q in zip(g, h))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", [(3, 64, 40), (4, 2048, 700)], ids=str)
def test_offsets_past_32_bits(size, dtype):
    """Rows of x, and then of W's transpose or of W, 2^31 + 8 (2^23 + 8) elements apart."""
    n, d, classes = size
    x, w, y, b = problem(*size, dtype, 21)
    want, wg = gmb.linear_loss(x, w, y, bias=b)
    apart = (1 << 31) + 8
    memory = torch.empty((n - 1) * apart + d, dtype=dtype, device="cuda")
    far = memory.as_strided((n, d), (apart, 1))
    far.copy_(x)
    loss, g = gmb.linear_loss(far, w, y, bias=b)
    assert torch.equal(loss, want) and all(torch.equal(p, q) for p, q in zip(g, wg))
    apart = (1 << 23) + 8                            # (700 rows of it: 5.9 billion elements)
    memory = torch.empty((classes - 1) * apart + d, dtype=dtype, device="cuda")
    far = memory.as_strided((classes, d), (apart, 1))
    far.copy_(w)
    loss, g = gmb.linear_loss(x, far, y, bias=b)
    assert torch.equal(loss, want) and all(torch.equal(p, q) for p, q in zip(g, wg))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_two_streams_at_once(dtype):
    problems = [problem(400, 96, 1500, dtype, 19), problem(250, 64, 900, dtype, 20)]
    want = [gmb.linear_loss(x, w, y, bias=b) for x, w, y, b in problems]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(5):
        for k, (x, w, y, b) in enumerate(problems):
            with torch.cuda.stream(streams[k]):
                got[k].append(gmb.linear_loss(x, w, y, bias=b))
    torch.cuda.synchronize()
    for k, (loss, g) in enumerate(want):
        for mine, h in got[k]:
            assert torch.equal(mine, loss) and all(torch.equal(p, q) for p, q in zip(g, h))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gradients_asked_for_one_by_one(dtype):
    x, w, y, b = problem(150, 96, 333, dtype, 3)
    loss, all_ = gmb.linear_loss(x, w, y, bias=b)
    for name in ("x", "w", "bias"):
        loss2, g = gmb.linear_loss(x, w, y, bias=b, grad=(name,))
        assert torch.equal(loss2, loss) and torch.equal(getattr(g, name), getattr(all_, name))
        assert sum(v is not None for v in g) == 1


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", HEADS + [(140, 70, 300)], ids=str)
def test_rows_without_a_label(size, dtype):
    """Whatever stands in them, and labels of any value outside the classes."""
    n, d, classes = size
    x, w, y, b = problem(n, d, classes, dtype, 4, none=0.0)
    off = torch.arange(n, device="cuda") % 3 == 1
    y[off] = torch.where(torch.arange(int(off.sum()), device="cuda") % 2 == 0, classes, -(1 << 31)).int()
    clean, cg = gmb.linear_loss(x, w, y, bias=b)
    check(x, w, y, b, clean, cg)
    dirty = x.clone()
    dirty[off] = float("nan")
    dirty[off.nonzero()[0, 0]] = float("inf")
    dirty[off.nonzero()[1, 0]] = torch.finfo(dtype).min
    loss, g = gmb.linear_loss(dirty, w, y, bias=b)
    assert torch.equal(loss, clean) and all(torch.equal(p, q) for p, q in zip(g, cg))
    assert not g.x[off].any()
    # none has one
    loss, g = gmb.linear_loss(dirty, w, torch.full_like(y, -1), bias=b)
    assert loss.item() == 0 and not any(v.any() for v in g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", HEADS, ids=str)
def test_classes_that_cannot_be(size, dtype):
    x, w, y, b = problem(*size, dtype, 5, none=0.0)
    b[::2] = -math.inf
    y = torch.randint(0, size[2] // 2, (size[0],), device="cuda", dtype=torch.int32) * 2 + 1
    loss, g = gmb.linear_loss(x, w, y, bias=b)
    check(x, w, y, b, loss, g)
    assert not g.w[::2].any() and not g.bias[::2].any()
    y[3] = 0                                     # the label cannot be: an infinite loss, a gradient all the same
    loss, g2 = gmb.linear_loss(x, w, y, bias=b)
    assert loss.item() == math.inf and bool(g2.x.isfinite().all())
    b[:] = -math.inf                             # nothing can be
    loss, g = gmb.linear_loss(x, w, y, bias=b)
    assert loss.item() == 0 and not any(v.any() for v in g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", HEADS, ids=str)
def test_not_numbers_stay_in_their_rows(size, dtype):
    x, w, y, b = problem(*size, dtype, 6, none=0.0)
    want, wg = gmb.linear_loss(x, w, y, bias=b)
    bad = x.clone()
    bad[7, 3] = float("nan")
    loss, g = gmb.linear_loss(bad, w, y, bias=b)
    assert math.isnan(loss.item()) and bool(g.x[7].isnan().all())
    keep = torch.arange(size[0], device="cuda") != 7
    assert torch.equal(g.x[keep], wg.x[keep])
    w[5, 5] = float("inf")
    assert not math.isfinite(gmb.linear_loss(x, w, y, bias=b)[0].item())


@pytest.mark.parametrize("size", HEADS, ids=str)
def test_sizes_of_values(size):
    """fp32 operands far from one, rows and weights of very different sizes."""
    for sx, sw in [(1e-12, 1e12), (1e15, 1e-16), (1e-30, 1e29), (1e-40, 1.0)]:
        x, w, y, b = problem(*size, torch.float32, 7)
        x, w = x * sx, w * sw
        loss, g = gmb.linear_loss(x, w, y, bias=b)
        check(x, w, y, b, loss, g)
    x, w, y, b = problem(*size, torch.float32, 8)
    x[::7] *= 1e-6
    x[1::7] *= 20
    loss, g = gmb.linear_loss(x, w, y, bias=b)
    check(x, w, y, b, loss, g)
    loss, g = gmb.linear_loss(torch.zeros_like(x), torch.zeros_like(w), y)
    check(torch.zeros_like(x), torch.zeros_like(w), y, None, loss, g)


@pytest.mark.parametrize("dtype, size", [(torch.bfloat16, (9000, 24, 30000)), (torch.float32, (5000, 40, 24001)),
                                         (torch.bfloat16, (200, 8, 900_000)), (torch.float32, (20_000, 16, 47))], ids=str)
def test_in_pieces(dtype, size):
    """More than 384 MB of gradients of logits: the classes in pieces, sums that are split."""
    x, w, y, b = problem(*size, dtype, 9)
    loss, g = gmb.linear_loss(x, w, y, bias=b)
    check(x, w, y, b, loss, g)
    if size[2] < 100_000:
        loss, g = gmb.linear_loss(x, w.t().contiguous().t(), y, bias=b)
        check(x, w, y, b, loss, g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_the_same_bits_every_time(dtype):
    for size in HEADS + [(300, 200, 3000)]:
        same_bits(*problem(*size, dtype, 10))


def same_bits(x, w, y, b):
    first, g = gmb.linear_loss(x, w, y, bias=b)
    for _ in range(3):
        loss, h = gmb.linear_loss(x, w, y, bias=b)
        assert torch.equal(loss, first) and all(torch.equal(p, q) for p, q in zip(g, h))


def test_no_rows():
    for dtype in TYPES:
        x, w, y, b = problem(0, 10, 33, dtype, 11)
        loss, g = gmb.linear_loss(x, w, y, bias=b)
        assert loss.item() == 0 and g.x.shape == (0, 10) and not g.w.any() and not g.bias.any()
        assert gmb.linear_loss(x, w, y, grad=False)[0].item() == 0


def test_gradients_against_differences():
    x, w, y, b = problem(4, 5, 9, torch.float32, 12, none=0.25)
    _, g = gmb.linear_loss(x, w, y, bias=b)
    h = 2.0 ** -6
    for t, grad, name in ((x, g.x, "x"), (w, g.w, "w"), (b, g.bias, "bias")):
        for i in range(t.numel()):
            at = t.view(-1)[i].item()
            value = []
            for s in (h, -h):
                t.view(-1)[i] = at + s
                value.append(gmb.linear_loss(x, w, y, bias=b, grad=False)[0].item())
            t.view(-1)[i] = at
            # h^2 / 6 of a third derivative (at most the operand cubed), a loss's own error over h
            size = max(float(x.abs().max()), float(w.abs().max()), 1.0) ** 3
            assert abs((value[0] - value[1]) / (2 * h) - grad.reshape(-1)[i].item()) <= h * h / 6 * size + 2 * REL * 4 / h, name


def test_captured_and_replayed_two_graphs_of_one_workspace():
    x, w, y, b = problem(300, 128, 1000, torch.float32, 13)
    x2, w2, y2, b2 = problem(77, 64, 2000, torch.bfloat16, 14)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    calls = [lambda: gmb.linear_loss(x, w, y, bias=b, workspace=ws), lambda: gmb.linear_loss(x2, w2, y2, bias=b2, workspace=ws)]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in calls:
            c()
    torch.cuda.current_stream().wait_stream(side)
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c())
        graphs.append(g)
    for k in range(4):
        x.mul_(0.9)
        x2.mul_(1.125)
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for c, (loss, grads) in zip(calls, outs):
            want, wg = c()
            assert torch.equal(loss, want) and all(torch.equal(p, q) for p, q in zip(grads, wg)), k


def test_on_another_stream():
    x, w, y, b = problem(500, 100, 700, torch.float32, 15)
    want, wg = gmb.linear_loss(x, w, y, bias=b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        loss, g = gmb.linear_loss(x, w, y, bias=b)
    side.synchronize()
    assert torch.equal(loss, want) and all(torch.equal(p, q) for p, q in zip(g, wg))


def test_refusals_of_the_binding():
    x, w, y, b = problem(8, 16, 20, torch.float32, 16)
    for call in [lambda: gmb.linear_loss(x.half(), w.half(), y), lambda: gmb.linear_loss(x, w.bfloat16(), y),
                 lambda: gmb.linear_loss(x, w[:, :8], y), lambda: gmb.linear_loss(x, w, y.long()),
                 lambda: gmb.linear_loss(x, w, y[:4]), lambda: gmb.linear_loss(x, w, y, bias=b[:3]),
                 lambda: gmb.linear_loss(x, w, y, bias=b.double()), lambda: gmb.linear_loss(x.cpu(), w, y),
                 lambda: gmb.linear_loss(x, w.cpu(), y), lambda: gmb.linear_loss(x.t(), w, y),
                 lambda: gmb.linear_loss(x, w, y, grad=("y",)), lambda: gmb.linear_loss(x, w, y, loss=torch.empty(2, device="cuda")),
                 lambda: gmb.linear_loss(x, w[0], y)]:
        with pytest.raises((TypeError, ValueError, gmb.GmbError)):
            call()
