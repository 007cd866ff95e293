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

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


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
