"""The norm's backward where a row's squares add up past fp32's range: the row norms
to 0, and what reaches its gradient is the carry alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import paper_2010_05337_amd as gmb  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("shape", [(5, 7), (33, 100), (40, 256), (9, 1025), (3, 8200), (2, 32769)], ids=str)
def test_rows_whose_squares_overflow(shape, dtype):
    n, dim = shape
    gen = torch.Generator().manual_seed(1)
    r, dy, carry = (torch.randn(n, dim, generator=gen).to(dtype).cuda() for _ in range(3))
    g = torch.ones(dim, device="cuda")
    r[1] = 3e38                                # (the products with dy add up past the range too)
    dy[1] = dy[1].abs() + 1
    y, _ = gmb.rms_norm(r, g, 1e-5)
    assert not y[1].any()
    d = gmb.Dropout(0.5, 3)
    got = gmb.rms_norm_backward(dy, r, g, 1e-5, carry=carry, dropout=d)
    assert torch.equal(got.residual[1], carry[1])
    assert torch.equal(got.x[1], gmb.dropout(carry, d)[1])
    # the other rows, and the weight's gradient, as without that row
    calm = r.clone()
    calm[1] = 0
    want = gmb.rms_norm_backward(dy, calm, g, 1e-5, carry=carry, dropout=d)
    others = torch.arange(n, device="cuda") != 1
    assert torch.equal(got.residual[others], want.residual[others]) and torch.equal(got.x[others], want.x[others])
    assert torch.equal(got.weight, want.weight)
