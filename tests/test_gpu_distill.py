"""The distillation loss and its gradient on the GPU against the definition in
64 bits.

Bounds: an exponential's argument passes two roundings and the instruction's
own, so with arguments down to -D (terms below 2^-30 of the sum apart, which
the sum's own rounding covers) it is off by (2 D + 4) half-steps at most; a
sum of positive terms adds a half-step for each addition of one thread's chain
and of the exchanges, and a quotient two more.  EPS below covers them with
D = 32 and chains of 64: relative to each of the parts that a gradient or a
loss is the sum of."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import mx_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402

U32, UBF16 = 2.0 ** -24, 2.0 ** -8
EPS = (2 * 32 + 4 + 64 + 16) * U32


def inputs(n, C, k, seed, dtype=torch.float32, spread=2.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.normal(size=(n, C)) * spread).astype(np.float32)).to(dtype)
    top = (rng.normal(size=(n, k)) * 2 + 3).astype(np.float32)
    cls = rng.integers(0, C, size=(n, k)).astype(np.int32)
    cls[rng.random(size=(n, k)) < 0.1] = -1
    if n > 3:
        cls[1] = -1                              # nothing of the teacher's
        top[2, : k // 2] = -np.inf               # some entries impossible
        cls[3] = cls[3, 0]                       # one class, often
    labels = rng.integers(0, C, size=n).astype(np.int32)
    labels[rng.random(size=n) < 0.2] = -1
    labels[0] = C
    return z, top, cls, labels


def parts(z, alpha, T, n, labels):
    """The gradient's parts' magnitudes beside the teacher's and the label's
    own (both at most alpha T / n and (1 - alpha) / n)."""
    m = z.max(axis=1, keepdims=True)
    qt = np.exp((z - m) / T)
    q = np.exp(z - m)
    g = alpha * T * qt / qt.sum(1, keepdims=True)
    if labels is not None:
        g = g + (1 - alpha) * q / q.sum(1, keepdims=True)
    return g / n


def check(z, top, cls, labels, alpha, T, want_grad=True):
    n, C = z.shape
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    loss, grad = gmb.distill_loss(z.cuda(), dev(top), dev(cls), labels=dev(labels), alpha=alpha, temperature=T,
                                  grad=want_grad)
    zh = z.float().numpy().astype(np.float64)
    ref, g, size = mx_ref.distill(zh, top, cls, labels, alpha, T)
    # a log-probability is off by EPS and by half-steps of its magnitude
    tol = (EPS * (size + alpha * T * T + 1) + n * U32 * size).mean() * 2
    assert abs(float(loss) - ref.mean()) <= tol, (float(loss), ref.mean(), tol)
    if not want_grad:
        assert grad is None
        return
    assert grad.dtype == z.dtype
    got = grad.double().cpu().numpy()
    bound = EPS * (parts(zh, alpha, T, n, labels) + np.abs(g))
    # the classes that the teacher or a label names: its shares' own errors
    for i in range(n):
        c = cls[i][(cls[i] >= 0) & (cls[i] < C)]
        np.add.at(bound[i], c, EPS * alpha * T / n)
        if labels is not None and 0 <= labels[i] < C:
            bound[i, labels[i]] += EPS * (1 - alpha) / n
    if z.dtype == torch.bfloat16:
        bound = bound + UBF16 * (np.abs(g) + bound) + 2.0 ** -134
    bound = bound + 2.0 ** -126                  # below the least normal number
    off = np.abs(got - g) - bound
    assert np.all(off <= 0), (off.max(), np.unravel_index(off.argmax(), off.shape))


SIZES = [(1, 1, 1), (5, 2, 1), (64, 8, 3), (100, 47, 8), (33, 172, 40), (7, 511, 5), (6, 512, 9), (5, 513, 30),
         (9, 1024, 64), (8, 1025, 17), (4, 4096, 256), (70, 4097, 20), (66, 8193, 3), (65, 32768, 10), (5, 5000, 9),
         (3, 33001, 100), (1, 131072, 1000), (4099, 47, 8)]


@pytest.mark.parametrize("n, C, k", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_loss_and_gradient(n, C, k, dtype):
    print(f"{n} rows of {C} classes, {k} entries, {dtype}", flush=True)
    z, top, cls, labels = inputs(n, C, k, n + C, dtype)
    check(z, top, cls, labels, 0.5, 2.0)


@pytest.mark.parametrize("n, C, k", [(40, 3, 3), (33, 50, 128), (20, 50, 129), (20, 60, 257), (37, 200, 255),
                                     (20, 200, 257), (9, 900, 512), (9, 900, 513), (70, 1000, 1024), (3, 40000, 1023),
                                     (5, 20000, 33), (9, 31000, 5)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_entries_beside_classes(n, C, k, dtype):
    """Entries by the ones, whole fours and more than classes (so that most of
    a class's entries add up)."""
    print(f"{n} rows of {C} classes, {k} entries, {dtype}", flush=True)
    z, top, cls, labels = inputs(n, C, k, n + k, dtype)
    check(z, top, cls, labels, 0.6, 1.5)


@pytest.mark.parametrize("alpha, T", [(0.0, 1.0), (1.0, 1.0), (0.3, 4.0), (0.9, 0.5), (1.0, 100.0), (0.25, 1.0)])
@pytest.mark.parametrize("C", [47, 3001, 40000])
@pytest.mark.parametrize("with_labels", [False, True])
def test_weights_and_temperatures(alpha, T, C, with_labels):
    z, top, cls, labels = inputs(6, C, 12, C)
    check(z, top, cls, labels if with_labels else None, alpha, T)


@pytest.mark.parametrize("C, dtype", [(1100, torch.float32), (4100, torch.bfloat16), (8190, torch.float32),
                                      (20003, torch.bfloat16), (20003, torch.float32), (32768, torch.float32)], ids=str)
def test_large_gradients(C, dtype):
    """Gradients past 64 MB: the rows are a few ones again and again, and each
    gets the gradient of the same row of a small batch (times their numbers)."""
    few = 8
    n = (1 << 26) // (C * (4 if dtype == torch.float32 else 2)) // few * few + few
    print(f"{n} rows of {C} {dtype}", flush=True)
    z, top, cls, labels = inputs(few, C, 5, C, dtype)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    rep = lambda a: a.repeat(n // few, *[1] * (a.dim() - 1))  # noqa: E731
    kw = dict(alpha=0.5, temperature=2.0)
    loss, grad = gmb.distill_loss(rep(z.cuda()), rep(dev(top)), rep(dev(cls)), labels=rep(dev(labels)), **kw)
    zh = z.float().numpy().astype(np.float64)
    ref, g, size = mx_ref.distill(zh, top, cls, labels, 0.5, 2.0)
    tol = (EPS * (size + 2.0 + 1) + n * U32 * size).mean() * 2
    assert abs(float(loss) - ref.mean()) <= tol
    bound = EPS * (parts(zh, 0.5, 2.0, few, labels) + np.abs(g) + (0.5 * 2.0 + 0.5) * 5 / few)
    if dtype == torch.bfloat16:
        bound = bound + UBF16 * (np.abs(g) + bound)
    got = grad.view(n // few, few, C).double() * (n / few)
    off = (got - torch.from_numpy(g).cuda()).abs() - torch.from_numpy(bound + 2.0 ** -100).cuda()
    assert float(off.max()) <= 0


def test_loss_alone():
    z, top, cls, labels = inputs(50, 60, 6, 1)
    check(z, top, cls, labels, 0.5, 2.0, want_grad=False)


@pytest.mark.parametrize("C", [40, 2000, 50000])
def test_masked_classes(C):
    """Logits of -inf (classes that cannot be), of the type's lowest value, and
    rows of nothing else."""
    z, top, cls, labels = inputs(8, C, 6, 5)
    z[:, ::3] = -np.inf
    z[1] = -np.inf
    z[2] = torch.finfo(torch.float32).min
    z[4, 1::3] = -1e30                           # a finite mask whose loss is finite too
    z[6, 1::3] = torch.finfo(torch.float32).min
    cls[6] = -1
    labels[:] = (labels // 3 * 3 + 1) % C        # a class that can be
    labels[labels % 3 == 0] = -1
    labels[6] = 2
    cls = np.where(cls % 3 == 0, -1, cls)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    loss, grad = gmb.distill_loss(z.cuda(), dev(top), dev(cls), labels=dev(labels), alpha=0.5, temperature=2.0)
    zh = z.numpy().astype(np.float64)
    got = grad.cpu().numpy()
    assert np.isfinite(got).all() and np.isfinite(float(loss))
    assert np.all(got[1] == 0) and np.all(got[:, ::3][np.isneginf(zh[:, ::3])] == 0)
    ref, g, _ = mx_ref.distill(zh, top, cls, labels, 0.5, 2.0)
    assert np.all(np.abs(got - g) <= EPS * (np.abs(g) + 2.0 * 0.5 / 8 + 0.5 / 8))
    assert abs(float(loss) - ref.mean()) <= 1e-5 * max(1.0, abs(ref.mean()))


@pytest.mark.parametrize("C", [40, 3000, 50000])
def test_what_is_no_number_stays_in_its_row(C):
    z, top, cls, labels = inputs(8, C, 6, 6)
    z[3, 5] = np.nan
    z[5, 7] = np.inf
    labels[:] = 1
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    loss, grad = gmb.distill_loss(z.cuda(), dev(top), dev(cls), labels=dev(labels), alpha=0.5, temperature=1.0)
    got = grad.cpu().numpy()
    assert np.isnan(float(loss)) and np.isnan(got[3]).all()
    assert np.isnan(got[5]).any()
    assert np.isfinite(got[[0, 1, 2, 4, 6, 7]]).all()


def test_an_impossible_class_that_the_teacher_wants():
    """The loss is infinite, the gradient finite."""
    z = torch.zeros(2, 10)
    z[0, 4] = -np.inf
    top, cls = np.zeros((2, 1), np.float32), np.array([[4], [4]], np.int32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    loss, grad = gmb.distill_loss(z.cuda(), dev(top), dev(cls), alpha=1.0)
    assert float(loss) == np.inf
    assert float(grad[0, 4]) == -0.5 and np.isfinite(grad.cpu().numpy()).all()


@pytest.mark.parametrize("C", [10, 40000])
@pytest.mark.parametrize("T", [0.25, 1.0, 8.0])
def test_a_teacher_of_the_lowest_value(C, T):
    """Rows whose teacher logits are all the type's lowest value (equal shares,
    also where the value over T is past the type), and some of them."""
    z, top, cls, labels = inputs(4, C, 5, 3)
    cls = np.tile(np.arange(5, dtype=np.int32), (4, 1))
    low = np.finfo(np.float32).min
    top[0] = low
    top[1, 1:] = low
    top[2, :] = [3e38, -3e38, 3e38, low, 0.0]
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    loss, grad = gmb.distill_loss(z.cuda(), dev(top), dev(cls), alpha=1.0, temperature=T)
    ref, g, size = mx_ref.distill(z.numpy().astype(np.float64), top.astype(np.float64), cls, None, 1.0, T)
    assert np.all(np.abs(grad.cpu().numpy() - g) <= EPS * (np.abs(g) + T / 4))
    assert abs(float(loss) - ref.mean()) <= (EPS * (size + T * T + 1)).mean() * 2


def test_more_rows_than_a_grid_counts():
    """2^28 + 3 rows of 16 threads are more than 32 bits count.  All rows are
    one of two, and a thread of the mean adds 2^16 terms: its sum is off by
    2^16 half-steps at most, and those of the rows by EPS each."""
    n = (1 << 28) + 3
    print(f"distill: {n} rows", flush=True)
    zero = torch.tensor([[0.0, 1.0], [2.0, 0.0]])
    z = torch.empty((n, 2), dtype=torch.bfloat16, device="cuda")
    z[0::2], z[1::2] = zero[0].cuda(), zero[1].cuda()
    top = torch.ones((n, 1), device="cuda")
    cls = torch.zeros((n, 1), dtype=torch.int32, device="cuda")
    loss, grad = gmb.distill_loss(z, top, cls, alpha=1.0)
    per, g, _ = mx_ref.distill(zero.double().numpy(), np.ones((2, 1)), np.zeros((2, 1), np.int32), None, 1.0, 1.0)
    want = ((n + 1) // 2 * per[0] + n // 2 * per[1]) / n
    assert abs(float(loss) - want) <= (2.0 ** 16 * U32 + EPS) * want
    got = torch.cat([grad[:2], grad[n // 2 - n // 2 % 2:][:2], grad[n - 3:n - 1]]).float().cpu().numpy()
    g = np.tile(g * 2 / n, (3, 1))               # (of two rows' mean there)
    assert np.all(np.abs(got - g) <= (UBF16 + EPS) * np.abs(g) + 2 * EPS / n)
    assert bool((grad.float().abs().amax(1) > 0).all())


def test_the_mean_of_many_rows():
    """2^26 rows of one loss: a running fp32 sum of 2^14 terms, each rounded the
    same way, would be off by up to 2^14 half-steps.  The mean is off by the
    row's own error and one rounding."""
    n = 1 << 26
    print(f"distill: {n} rows", flush=True)
    z = torch.empty((n, 2), dtype=torch.bfloat16, device="cuda")
    z[:, 0], z[:, 1] = 0.0, 1.0
    loss, _ = gmb.distill_loss(z, torch.ones((n, 1), device="cuda"),
                               torch.zeros((n, 1), dtype=torch.int32, device="cuda"), alpha=1.0, grad=False)
    per, _, _ = mx_ref.distill(np.array([[0.0, 1.0]]), np.ones((1, 1)), np.zeros((1, 1), np.int32), None, 1.0, 1.0)
    assert abs(float(loss) - per[0]) <= (EPS + U32) * per[0], (float(loss), per[0])


def test_more_threads_than_a_grid_counts():
    """2^29 + 3 rows of two classes: 8 threads each are more than 32 bits count.
    All rows are one of two kinds; the mean adds one rounding."""
    n = (1 << 29) + 3
    print(f"distill: {n} rows", flush=True)
    kinds = torch.tensor([[0.0, 1.0], [2.0, 0.0]])
    z = torch.empty((n, 2), dtype=torch.bfloat16, device="cuda")
    z[0::2], z[1::2] = kinds[0].cuda(), kinds[1].cuda()
    loss, grad = gmb.distill_loss(z, torch.ones((n, 1), device="cuda"),
                                  torch.zeros((n, 1), dtype=torch.int32, device="cuda"), alpha=1.0)
    per, g, _ = mx_ref.distill(kinds.double().numpy(), np.ones((2, 1)), np.zeros((2, 1), np.int32), None, 1.0, 1.0)
    want = ((n + 1) // 2 * per[0] + n // 2 * per[1]) / n
    assert abs(float(loss) - want) <= (EPS + U32) * want
    # the rows of a kind have the same bits, and those are near the definition's
    assert bool((grad[0:n - 1:2] == grad[0]).all()) and bool((grad[1::2] == grad[1]).all())
    assert bool((grad[n - 1] == grad[0]).all())
    got, g = grad[:2].double().cpu().numpy(), g * 2 / n
    assert np.all(np.abs(got - g) <= (UBF16 + EPS) * np.abs(g) + 2 * EPS / n)


def test_the_gradient_is_the_loss_s_difference():
    """Central differences of the GPU's own loss (fp32: steps of 2^-5 and a
    bound of the differences' second order and rounding)."""
    z, top, cls, labels = inputs(2, 6, 3, 9, spread=1.0)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    run = lambda t: gmb.distill_loss(t.cuda(), dev(top), dev(cls), labels=dev(labels), alpha=0.6, temperature=1.5)  # noqa: E731
    grad = run(z)[1].cpu().numpy()
    h = 2.0 ** -5
    for i in range(2):
        for c in range(6):
            a, b = z.clone(), z.clone()
            a[i, c] += h
            b[i, c] -= h
            d = (float(run(a)[0]) - float(run(b)[0])) / (2 * h)
            # third derivative of log-sum-exp is at most 1 (over T^2, times T^2 / n)
            assert abs(d - grad[i, c]) <= h * h / 6 + 1e-4


def test_streams_graphs_and_given_buffers():
    z, top, cls, labels = inputs(40, 9000, 8, 2)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    zc, topc, clsc, yc = z.cuda(), dev(top), dev(cls), dev(labels)
    grad, loss = torch.empty_like(zc), torch.empty(1, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    kw = dict(labels=yc, alpha=0.4, temperature=2.0, grad=grad, loss=loss, workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gmb.distill_loss(zc, topc, clsc, **kw)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gmb.distill_loss(zc, topc, clsc, **kw)
    for seed in (3, 4, 5):
        y = inputs(40, 9000, 8, seed)[0].cuda()
        want_loss, want = gmb.distill_loss(y, topc, clsc, labels=yc, alpha=0.4, temperature=2.0)
        zc.copy_(y)
        grad.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, want) and torch.equal(loss, want_loss)


def test_refusals():
    z, top, cls, labels = (torch.from_numpy(a).cuda() if isinstance(a, np.ndarray) else a.cuda()
                           for a in inputs(5, 20, 4, 1))
    for call in (lambda: gmb.distill_loss(z.half(), top, cls), lambda: gmb.distill_loss(z[0], top, cls),
                 lambda: gmb.distill_loss(z.t(), top, cls), lambda: gmb.distill_loss(z, top.double(), cls),
                 lambda: gmb.distill_loss(z, top, cls.long()), lambda: gmb.distill_loss(z, top[:4], cls[:4]),
                 lambda: gmb.distill_loss(z, top, cls[:, :3]), lambda: gmb.distill_loss(z, top, cls, labels=labels[:4]),
                 lambda: gmb.distill_loss(z, top, cls, labels=labels.long()),
                 lambda: gmb.distill_loss(z, top, cls, grad=z), lambda: gmb.distill_loss(z, top, cls, alpha=2.0),
                 lambda: gmb.distill_loss(z, top, cls, temperature=0.0),
                 lambda: gmb.distill_loss(z, top[:, :0].contiguous(), cls[:, :0].contiguous()),
                 lambda: gmb.distill_loss(z, top, cls, loss=torch.empty(2, device="cuda"))):
        with pytest.raises((TypeError, ValueError, gmb.GmbError)):
            call()
    loss, grad = gmb.distill_loss(z[:0], top[:0], cls[:0])
    assert float(loss) == 0 and grad.shape == (0, 20)
