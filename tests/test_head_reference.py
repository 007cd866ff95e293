"""The 64-bit definitions of dropout, the norm and the cross-entropy over many
classes (head_ref.py) themselves: Philox's published answers, gradients against
differences, rows without a label (CPU)."""
import numpy as np
import pytest
import torch

import head_ref


@pytest.mark.parametrize("counter, key, want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_published_answers(counter, key, want):
    assert tuple(int(w) for w in head_ref.philox(*counter, *key)) == want


def test_keep_rate_and_independence():
    k = head_ref.keep(np.arange(2000), 512, 0.3, 7).numpy()
    n = k.size
    p = head_ref.threshold(0.3) / 65536
    assert abs(k.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)
    other = head_ref.keep(np.arange(2000), 512, 0.3, 7, layer=1).numpy()
    both = (k & other).mean()
    q = (1 - p) ** 2
    assert abs(both - q) < 5 * np.sqrt(q * (1 - q) / n)
    assert head_ref.keep([5], 9, 0.0, 1).all() and not head_ref.keep([5], 9, 1.0, 1).any()
    # a row's mask goes with its key
    assert torch.equal(head_ref.keep([9, 3, 9], 40, 0.5, 3)[0], head_ref.keep([1, 2, 9], 40, 0.5, 3)[2])


def _differences(f, x, h=1e-5):
    g = torch.zeros_like(x)
    for i in range(x.numel()):
        a, b = x.clone(), x.clone()
        a.view(-1)[i] += h
        b.view(-1)[i] -= h
        g.view(-1)[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_norm_gradients_are_differences():
    gen = torch.Generator().manual_seed(1)
    r, dy, carry = (torch.randn(4, 7, generator=gen, dtype=torch.float64) for _ in range(3))
    w = torch.randn(7, generator=gen, dtype=torch.float64)
    f = lambda r, w: (head_ref.rms_norm(r, w, 0.1) * dy).sum() + (r * carry).sum()  # noqa: E731
    dr, dw = head_ref.rms_norm_backward(dy, r, w, 0.1, carry)
    # (central differences: the third derivative's h^2 / 6 and a rounding over h)
    assert torch.allclose(dr, _differences(lambda a: f(a, w), r), atol=1e-8)
    assert torch.allclose(dw, _differences(lambda a: f(r, a), w), atol=1e-8)


def test_loss_gradients_are_differences():
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(5, 3, generator=gen, dtype=torch.float64)
    w = torch.randn(6, 3, generator=gen, dtype=torch.float64)
    b = torch.randn(6, generator=gen, dtype=torch.float64)
    y = torch.tensor([0, 5, -1, 2, 6], dtype=torch.int32)
    loss, dx, dw, db = head_ref.linear_loss(x, w, y, b)
    want = torch.nn.functional.cross_entropy((x @ w.t() + b)[[0, 1, 3]], y[[0, 1, 3]].long(), reduction="sum") / 5
    assert abs(loss - want) < 1e-12
    assert torch.allclose(dx, _differences(lambda a: head_ref.linear_loss(a, w, y, b)[0], x), atol=1e-8)
    assert torch.allclose(dw, _differences(lambda a: head_ref.linear_loss(x, a, y, b)[0], w), atol=1e-8)
    assert torch.allclose(db, _differences(lambda a: head_ref.linear_loss(x, w, y, a)[0], b), atol=1e-8)


def test_rows_without_anything():
    x = torch.full((2, 3), float("nan"), dtype=torch.float64)
    w = torch.ones(4, 3, dtype=torch.float64)
    loss, dx, dw, db = head_ref.linear_loss(x, w, torch.tensor([-1, 4], dtype=torch.int32))
    assert loss == 0 and not dx.any() and not dw.any() and not db.any()
    b = torch.full((4,), -np.inf, dtype=torch.float64)
    loss, dx, dw, db = head_ref.linear_loss(torch.ones(2, 3, dtype=torch.float64), w, torch.tensor([0, 1], dtype=torch.int32), b)
    assert loss == 0 and not dx.any() and not dw.any() and not db.any()
