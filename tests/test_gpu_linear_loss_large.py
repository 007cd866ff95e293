"""The cross-entropy over many classes where its sums are long, its classes come
in many pieces and its weights are read as they lie.

Bounds of the long sums, in half-steps U = 2^-24.  The logits of all classes but
one are equal, so everything has a closed form in 64 bits.  A logit's error DZ
is its products' and sum's ((3 d + 10) U of their size, at most 1 here, and
2^-22 of it in fp32) and its bias's (2 U of the bias).  A row's sum of
exponentials: an argument below 16 in magnitude 26 U, its exponential 2, a
tile's chain at most 31, the joined lanes, waves and chunks (at most 48 links of
two roundings a factor and one a sum, of which a link passes on the larger part)
144: SUM = 203 U.  The logarithm and what it is added to are at most 40 in powers
of two: 2 x 40 U.  So a loss is off by 2 DZ + 283 U, a probability by that and
its own argument's, 2 DZ + 400 U of it, and a sum of it over the rows by another
64 U (registers, exchanges, 16 parts' chains)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import paper_2010_05337_amd as gmb  # noqa: E402
from test_gpu_linear_loss import check, problem  # noqa: E402

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
GUARD = 4096


# tiles of 256 x 256 in one chunk of the classes a row; W as it lies, in 256 chunks
@pytest.mark.parametrize("rows, d, classes, most, dtype", [
    (33_024, 8, 400_000, 8.0, torch.bfloat16), (33_024, 8, 400_000, 8.0, torch.float32),
    (33_024, 8, 200_000, 5.3, torch.bfloat16), (4, 1, 1 << 27, 6.3, torch.float32)], ids=str)
def test_long_sums_of_equal_exponentials(rows, d, classes, most, dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, d, device="cuda", generator=gen).to(dtype)
    w = torch.zeros(classes, d, device="cuda", dtype=dtype)
    w += (0.1 * torch.randn(d, device="cuda", generator=gen)).to(dtype)
    b = torch.zeros(classes, device="cuda")
    b[0] = most
    y = (torch.arange(rows, device="cuda") % 5).int()         # (classes 0 .. 4)
    top = float(b[0].double())
    total = math.exp(top) + classes - 1
    size = float((x.double().abs() @ w[0].double().abs()).max())
    dz = ((3 * d + 10) * U + 2.0 ** -22) * size + 2 * U * top
    want = math.log(total) - top * int((y == 0).sum()) / rows
    tol = 2 * dz + 283 * U
    for grad in (False, ("bias",)):
        loss, g = gmb.linear_loss(x, w, y, bias=b, grad=grad)
        err = abs(float(loss.double()) - want)
        assert err <= tol, ("loss", err, tol)
    p = 1 / total
    tol = (2 * dz + 464 * U) * p
    err = float((g.bias[5:].double() - p).abs().max())
    assert err <= tol, ("dbias", err / p, tol / p)
    err = abs(float(g.bias[0].double()) - (math.exp(top) / total - int((y == 0).sum()) / rows))
    assert err <= tol / p * math.exp(top) / total + 64 * U, ("dbias of the largest", err)


def guarded(bytes_, dtype, shape):
    """Memory of exactly that size, and the bytes behind it."""
    raw = torch.full((bytes_ + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
    assert raw.data_ptr() % 256 == 0
    return raw[:bytes_].view(dtype).view(shape), raw[bytes_:]


def through_the_abi(x, w, y, b, turned, names="xwb"):
    """(loss, LinearGrads) with a workspace of exactly the bytes asked for; nothing behind it or the results is written."""
    (n, d), classes, code = x.shape, w.shape[0], gmb._dtype_code(x.dtype)
    es = x.element_size()
    dx, gx = guarded(n * d * es, x.dtype, (n, d)) if "x" in names else (None, None)
    dw, gw = guarded(classes * d * es, x.dtype, (d, classes) if turned else (classes, d)) if "w" in names else (None, None)
    db, gb = guarded(classes * 4, torch.float32, (classes,)) if "b" in names and b is not None else (None, None)
    loss, gl = guarded(4, torch.float32, (1,))
    head = gmb.LinearHeadStruct(x.data_ptr(), x.stride(0), w.data_ptr(), *w.stride(), None if b is None else b.data_ptr(),
                                y.data_ptr(), n, d, classes, code, 0)
    grads = gmb.LinearGradsStruct(*[None if t is None else t.data_ptr() for t in (dx, dw, db)], int(turned), 0)
    need = gmb.lib().gmb_linear_loss_workspace_bytes(head, grads)
    ws, gs = guarded(need, torch.uint8, (need,))
    assert gmb.lib().gmb_linear_loss(head, grads, loss.data_ptr(), ws.data_ptr(), need, gmb._stream_handle()) == 0
    for name, guard in (("dx", gx), ("dw", gw), ("dbias", gb), ("loss", gl), ("workspace", gs)):
        assert guard is None or bool((guard == 0x5A).all()), name
    return loss, gmb.LinearGrads(dx, dw.t() if turned and dw is not None else dw, db)


# small heads, one tile, few rows over many classes, tiles of 64 and 256, sums that are split; and pieces of the classes
SIZES = [(1, 1, 1), (300, 65, 47), (1000, 256, 47), (5, 100, 20_001), (16, 100, 30_001), (129, 128, 257), (1500, 48, 172),
         (784, 63, 4133), (2100, 64, 5001), (9000, 24, 30_001), (5000, 64, 50_003)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_nothing_is_written_behind_the_workspace_and_the_results(size, dtype):
    x, w, y, b = problem(*size, dtype, 31)
    for turned in (False, True):
        loss, g = through_the_abi(x, w, y, b, turned)
        want, h = gmb.linear_loss(x, w, y, bias=b)
        assert torch.equal(loss, want) and torch.equal(g.x, h.x) and torch.equal(g.bias, h.bias)
        if not turned:
            check(x, w, y, b, loss, g)
            assert torch.equal(g.w, h.w)
        else:                                      # (the product's other operand order: the same sums)
            check(x, w, y, b, loss, g)


@pytest.mark.parametrize("d", [64, 192])
@pytest.mark.parametrize("bias", [False, True])
def test_pieces_of_weights_read_as_they_lie(d, bias):
    """bf16 rows of whole stages, at a stride past them, the classes in several pieces and the last one ragged."""
    n, classes = 9000, 30_001
    x, w, y, b = problem(n, d, classes, torch.bfloat16, 32, bias)
    wide = torch.full((classes, d + 64), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:, :d] = w
    view = wide[:, :d]
    for turned in (False, True):
        loss, g = through_the_abi(x, view, y, b, turned)
        check(x, w, y, b, loss, g)
        want, h = gmb.linear_loss(x, w, y, bias=b)
        assert torch.equal(loss, want) and torch.equal(g.x, h.x)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("names", ["w", "b", "x", "wb"])
def test_some_gradients_of_pieces(names, dtype):
    x, w, y, b = problem(9000, 24, 30_001, dtype, 33)
    want, h = gmb.linear_loss(x, w, y, bias=b)
    loss, g = through_the_abi(x, w, y, b, False, names)
    assert torch.equal(loss, want)
    check(x, w, y, b, loss, g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", [(60, 40, 200), (5, 100, 20_001), (60, 140, 1000), (2100, 64, 5000)], ids=str)
def test_a_mask_of_the_lowest_value_is_one_of_infinities(size, dtype):
    n, d, classes = size
    x, w, y, b = problem(n, d, classes, dtype, 34, none=0.0)
    lowest = torch.finfo(torch.float32).min
    for off, label in ((slice(0, None, 2), 1), (slice(0, None, 2), 0), (slice(0, None), 1)):   # (other classes, the labels too, all)
        y = torch.randint(0, classes // 2, (n,), device="cuda", dtype=torch.int32) * 2 + label
        never, low = b.clone(), b.clone()
        never[off], low[off] = -math.inf, lowest
        want, h = gmb.linear_loss(x, w, y, bias=never)
        loss, g = gmb.linear_loss(x, w, y, bias=low)
        assert torch.equal(loss, want) and all(torch.equal(p, q) for p, q in zip(g, h))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", [(60, 40, 20), (60, 40, 200), (5, 100, 20_001), (60, 140, 1000), (2100, 64, 5000)], ids=str)
def test_logits_far_from_zero(size, dtype):
    """Equal logits of any size: uniform probabilities (the bounds above; here arguments are 0)."""
    n, d, classes = size
    gen = torch.Generator(device="cuda").manual_seed(35)
    x = torch.randn(n, d, device="cuda", generator=gen).to(dtype)
    w = torch.zeros(classes, d, device="cuda", dtype=dtype)
    w += (0.1 * torch.randn(d, device="cuda", generator=gen)).to(dtype)
    y = (torch.arange(n, device="cuda") % 5).int()
    count = torch.bincount(y.long(), minlength=classes).double() / n
    for at in (1e5, -1e5, 1e9, -1e9, -1e30, 3e37, -2e38):
        b = torch.full((classes,), at, device="cuda")
        alone, _ = gmb.linear_loss(x, w, y, bias=b, grad=False)
        loss, g = gmb.linear_loss(x, w, y, bias=b)
        assert torch.equal(alone, loss)
        err = abs(float(loss.double()) - math.log(classes))
        assert err <= 283 * U, (at, "loss", err)
        err = float((g.bias.double() - (1 / classes - count)).abs().max())
        assert err <= 464 * U / classes + 64 * U * float(count.max()), (at, "dbias", err)
        # softmax - onehot times equal rows: nothing but its roundings, those of the entries (bf16: 2^-8 of each, their
        # magnitudes add up to 2) and of the sum of three part products a class, each addition a half-step of at most 2
        entry = 2 / n * ((2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -20) + 3 * (classes + 8) * U)
        assert float(g.x.abs().max()) <= entry * float(w[0].abs().max()), (at, "dx", float(g.x.abs().max()))
