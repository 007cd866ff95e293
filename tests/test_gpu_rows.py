"""Dropout and the root-mean-square norm on the GPU against their definitions in
64 bits.

Bounds, in half-steps U of fp32 (and one of bf16 for a result of that type): a
dropped-out value passes two roundings (the factor's and the product's), a sum
one more.  A row's sum of squares is a chain of at most 64 additions in a
thread, 6 exchanges and 16 waves: 86 U, with the mean and eps 90; its inverse
root half of that and the instruction's and Newton step's 6: INV = 51 U, a norm
two products more.  A second sum of the backward has 86 U of its terms'
magnitudes; the product of four such factors stays below 300 U."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import head_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U32 = U[torch.float32]
TYPES = [torch.float32, torch.bfloat16]
# rows: none to many; columns: one, around a piece, a wave's, every shape of the kernels, past what registers hold
SHAPES = [(1, 1), (5, 7), (3, 8), (70, 9), (64, 16), (33, 33), (257, 100), (40, 128), (19, 130), (300, 256), (9, 257), (7, 513),
          (4, 1025), (6, 2047), (5, 2049), (3, 4097), (3, 8192), (2, 8200), (2, 16392), (2, 32769), (1, 65536)]
EPS = 1e-5


def rows(n, dim, seed, dtype, pad=0):
    """Rows of several sizes, at a stride of dim + pad, and their values in 64 bits."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(n, dim, generator=gen) * torch.exp(torch.randn(n, 1, generator=gen))
    buf = torch.full((n, dim + pad), 77.0).to(dtype)
    buf[:, :dim] = x.to(dtype)
    return buf.cuda()[:, :dim]


def wide(t):
    return t.double().cpu()


def near(got, want, tol, what):
    got = wide(got)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((got - want).abs()[bad].max()), bad.nonzero()[:3].tolist())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_dropout(shape, dtype):
    n, dim = shape
    x, res = rows(n, dim, 1, dtype, pad=3), rows(n, dim, 2, dtype, pad=5)
    ids = torch.randint(0, 1 << 31, (n,), dtype=torch.int64, generator=torch.Generator().manual_seed(3)).int()
    for p, seed, layer, keys, add in [(0.5, 11, 0, None, None), (0.1, (1 << 63) + 5, 7, ids, res), (0.9, 12, 3, ids, None)]:
        d = gmb.Dropout(p, seed, layer)
        got = gmb.dropout(x, d, ids=None if keys is None else keys.cuda(), residual=add)
        kept = head_ref.keep(np.arange(n) if keys is None else keys.numpy(), dim, p, seed, layer)
        want = head_ref.drop(wide(x), kept, p)
        tol = 2 * U32 * want.abs()
        if add is not None:
            want = want + wide(add)
            tol = tol + U32 * want.abs()
        near(got, want, 1.001 * tol + U[dtype] * (want.abs() + tol) * (dtype is torch.bfloat16), (p, layer))
        if add is None:
            assert torch.equal(got.cpu() != 0, kept & (x.cpu() != 0))
        # the gradient: the same call
        assert torch.equal(gmb.dropout(x, d, ids=None if keys is None else keys.cuda()),
                           gmb.dropout(x, d, ids=None if keys is None else keys.cuda()))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_dropout_ends_of_p_and_what_is_dropped(dtype):
    x = rows(40, 70, 4, dtype)
    assert torch.equal(gmb.dropout(x, gmb.Dropout(0.0, 1)), x)
    assert not gmb.dropout(x, gmb.Dropout(1.0, 1)).any()
    kept = head_ref.keep(np.arange(40), 70, 0.5, 9)
    bad = x.clone()
    bad[~kept.cuda()] = float("nan")
    bad[0][~kept[0].cuda()] = float("inf")
    got = gmb.dropout(bad, gmb.Dropout(0.5, 9))
    assert torch.equal(got, gmb.dropout(x, gmb.Dropout(0.5, 9)))
    # in place, of x and of the residual
    want = gmb.dropout(x, gmb.Dropout(0.5, 9), residual=bad)
    y = x.clone()
    assert gmb.dropout(y, gmb.Dropout(0.5, 9), residual=bad, out=y) is y
    assert torch.equal(y, want) or torch.equal(y.nan_to_num(), want.nan_to_num())
    y = bad.clone()
    gmb.dropout(x, gmb.Dropout(0.5, 9), residual=y, out=y)
    assert torch.equal(y.nan_to_num(), want.nan_to_num())


def test_dropout_step_on_the_device():
    x = rows(50, 64, 5, torch.float32)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = gmb.Dropout(0.5, 21, 2, step=step)
    seen = []
    for k in (0, 1, -1):
        step.fill_(k)
        got = gmb.dropout(x, d)
        assert torch.equal(got.cpu() != 0, head_ref.keep(np.arange(50), 64, 0.5, 21, 2, step=k))
        seen.append(got)
    assert not torch.equal(seen[0], seen[1])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [0, 1, 33, 64])
def test_rows_behind_the_count_stay(n, dtype):
    x, res, g = rows(64, 100, 6, dtype), rows(64, 100, 7, dtype), torch.rand(100, device="cuda")
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    d = gmb.Dropout(0.5, 3)
    mark = torch.full_like(x, 5.0)
    got = gmb.dropout(x, d, residual=res, out=mark.clone(), count=count)
    assert torch.equal(got[:n], gmb.dropout(x, d, residual=res)[:n]) and bool((got[n:] == 5).all())
    y, r = gmb.rms_norm(x, g, EPS, residual=res, dropout=d, out=mark.clone(), sum_out=mark.clone(), count=count)
    y0, r0 = gmb.rms_norm(x, g, EPS, residual=res, dropout=d)
    assert torch.equal(y[:n], y0[:n]) and bool((y[n:] == 5).all())
    assert torch.equal(r[:n], r0[:n]) and bool((r[n:] == 5).all())
    for bits in (4, 8):
        rec = torch.full((64, gmb.mx_row_bytes(100, bits) + 16), 9, dtype=torch.uint8, device="cuda")
        gmb.rms_norm(x, g, EPS, residual=res, dropout=d, bits=bits, out=rec, count=count)
        w = gmb.mx_row_bytes(100, bits)
        assert bool((rec[n:] == 9).all()) and bool((rec[:, w:] == 9).all())
        assert torch.equal(rec[:n, :w], gmb.rms_norm(x, g, EPS, residual=res, dropout=d, bits=bits)[0][:n])
    grads = gmb.rms_norm_backward(y0, r0, g, EPS, dropout=d, count=count)
    if n:
        want = gmb.rms_norm_backward(y0[:n].contiguous(), r0[:n].contiguous(), g, EPS, dropout=d)
        assert torch.equal(grads.x[:n], want.x) and torch.equal(grads.residual[:n], want.residual)
        # (other workgroups: another order of the sums)
        assert torch.allclose(grads.weight, want.weight, rtol=1e-4, atol=1e-4)
    else:
        assert not grads.weight.any()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm(shape, dtype):
    n, dim = shape
    x, res = rows(n, dim, 8, dtype, pad=1), rows(n, dim, 9, dtype)
    g = torch.randn(dim, generator=torch.Generator().manual_seed(10)).cuda()
    low = dtype is torch.bfloat16
    for add, d, weight in [(None, None, g), (res, None, None), (res, gmb.Dropout(0.25, 77, 1), g), (None, gmb.Dropout(0.5, 78), g)]:
        y, r = gmb.rms_norm(x, weight, EPS, residual=add, dropout=d)
        want = wide(x)
        if d is not None:
            want = head_ref.drop(want, head_ref.keep(np.arange(n), dim, d.p, d.seed, d.layer), d.p)
        tol = 2 * U32 * want.abs()
        if add is not None:
            want = want + wide(add)
            tol = tol + U32 * want.abs()
        if add is None and d is None:
            assert r is x
        else:
            near(r, want, 1.001 * tol + U[dtype] * (want.abs() + tol) * low, "sum")
        want = head_ref.rms_norm(wide(r), None if weight is None else wide(weight), EPS)
        near(y, want, 64 * U32 * want.abs() + U[dtype] * (1 + 64 * U32) * want.abs() * low, "norm")
        # records: what the store's own quantisation makes of the fp32 norm of the same sums
        y32, _ = gmb.rms_norm(r.float().contiguous(), weight, EPS)
        for bits in (4, 8):
            rec, r2 = gmb.rms_norm(x, weight, EPS, residual=add, dropout=d, bits=bits)
            assert torch.equal(r2, r)
            assert torch.equal(rec, gmb.mx_quantise(y32, bits)), bits


def test_norm_rows_of_zeros_and_not_numbers():
    for dim in (100, 9000, 20000):
        x = rows(6, dim, 11, torch.float32)
        x[1] = 0
        x[2, 3] = float("nan")
        x[3, dim - 1] = float("inf")
        y, _ = gmb.rms_norm(x, None, EPS)
        assert not y[1].any() and bool(y[2].isnan().all()) and bool(y[3, dim - 1].isnan())
        other, _ = gmb.rms_norm(x[4:].contiguous(), None, EPS)
        assert torch.equal(y[4:], other)
        rec, _ = gmb.rms_norm(x, None, EPS, bits=8)
        assert torch.equal(gmb.mx_gather(None, rec, dim, 8)[1], torch.zeros(dim, device="cuda"))


def test_norm_of_the_smallest_eps():
    """2^-126 beside rows of zeros, and of values whose squares are 0 or no normal numbers."""
    eps = 2.0 ** -126
    x = torch.ones(4, 100, device="cuda") * torch.tensor([0.0, 1e-30, 1e-19, 3e-19], device="cuda")[:, None]
    y, _ = gmb.rms_norm(x, None, eps)
    want = head_ref.rms_norm(wide(x), torch.ones(100, dtype=torch.float64), eps)
    # (a square below 2^-126 is off by half of 2^-149: 2^-24 of eps)
    near(y, want, 64 * U32 * want.abs(), "norm")
    g = gmb.rms_norm_backward(torch.full_like(x, 1e-20), x, None, eps)
    assert bool(g.x.isfinite().all())


def test_norm_in_place():
    for dim in (256, 5000, 40000):
        x, res, g = rows(5, dim, 12, torch.float32), rows(5, dim, 13, torch.float32), torch.rand(dim, device="cuda")
        d = gmb.Dropout(0.5, 5)
        want, total = gmb.rms_norm(x, g, EPS, residual=res, dropout=d)
        a = res.clone()
        y, r = gmb.rms_norm(x, g, EPS, residual=a, dropout=d, sum_out=a)
        assert r is a and torch.equal(a, total) and torch.equal(y, want)
        a, b = x.clone(), res.clone()
        y, r = gmb.rms_norm(a, g, EPS, residual=b, dropout=d, sum_out=b, out=a)
        assert y is a and torch.equal(a, want) and torch.equal(b, total)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES + [(5000, 40), (3000, 300)], ids=str)
def test_norm_backward(shape, dtype):
    n, dim = shape
    low = dtype is torch.bfloat16
    r, dy, carry = rows(n, dim, 14, dtype, pad=2), rows(n, dim, 15, dtype, pad=7), rows(n, dim, 16, dtype)
    g = torch.randn(dim, generator=torch.Generator().manual_seed(17)).cuda()
    R, D, G = wide(r), wide(dy), wide(g)
    for weight, add, d in [(g, None, None), (None, carry, None), (g, carry, gmb.Dropout(0.5, 99, 4))]:
        got = gmb.rms_norm_backward(dy, r, weight, EPS, carry=add, dropout=d)
        W = None if weight is None else G
        dr, dw = head_ref.rms_norm_backward(D, R, W, EPS, None if add is None else wide(add))
        s = 1 / torch.sqrt(R.square().mean(1, keepdim=True) + EPS)
        a = (D if W is None else D * W).abs()
        tol = 300 * U32 * s * (a + R.abs() * s * s * (a * R.abs()).mean(1, keepdim=True)) + U32 * dr.abs()
        near(got.residual, dr, tol + U[dtype] * (dr.abs() + tol) * low, "residual")
        if weight is None:
            assert got.weight is None
        else:
            # 58 U a term, a chain of at most 5 rows a thread, 64 rows and 128 parts
            near(got.weight, dw, 256 * U32 * (D * R * s).abs().sum(0), "weight")
        if d is None:
            assert got.x is got.residual
        else:
            kept = head_ref.keep(np.arange(n), dim, d.p, d.seed, d.layer)
            want, by = head_ref.drop(dr, kept, d.p), 65536 / (65536 - head_ref.threshold(d.p))
            tol = torch.where(kept, by * tol + 2 * U32 * want.abs(), torch.zeros_like(tol))
            near(got.x, want, tol + U[dtype] * (want.abs() + tol) * low, "x")
        again = gmb.rms_norm_backward(dy, r, weight, EPS, carry=add, dropout=d)
        assert torch.equal(again.residual, got.residual) and (weight is None or torch.equal(again.weight, got.weight))


def test_norm_gradients_against_differences():
    n, dim = 3, 11
    x, dy, g = rows(n, dim, 18, torch.float32), rows(n, dim, 19, torch.float32), torch.rand(dim, device="cuda") + 0.5
    d = gmb.Dropout(0.5, 42, 1)
    got = gmb.rms_norm_backward(dy, gmb.rms_norm(x, g, 0.5, dropout=d)[1], g, 0.5, dropout=d)

    def value(x):
        return float((gmb.rms_norm(x, g, 0.5, dropout=d)[0].double() * dy.double()).sum())

    h = 2.0 ** -6
    for i in range(n):
        for j in range(dim):
            a, b = x.clone(), x.clone()
            a[i, j] += h
            b[i, j] -= h
            # the difference's own error: h^2 / 6 of a third derivative, 64 U of a row's sum over h
            row = float((gmb.rms_norm(x, g, 0.5, dropout=d)[0].double() * dy.double())[i].abs().sum())
            assert abs((value(a) - value(b)) / (2 * h) - float(got.x[i, j])) <= 200 * h * h * (1 + row) / 6 + 64 * U32 * row / h


def test_no_rows():
    x, g = torch.empty(0, 9, device="cuda"), torch.ones(9, device="cuda")
    assert gmb.dropout(x, gmb.Dropout(0.5, 1)).shape == (0, 9)
    assert gmb.rms_norm(x, g)[0].shape == (0, 9)
    got = gmb.rms_norm_backward(x, x, g)
    assert got.x.shape == (0, 9) and not got.weight.any()


def test_refusals_of_the_binding():
    x, d, g = rows(4, 8, 20, torch.float32), gmb.Dropout(0.5, 1), torch.ones(8, device="cuda")
    for call in [lambda: gmb.Dropout(1.5, 1), lambda: gmb.Dropout(0.5, 1, layer=-1), lambda: gmb.dropout(x.half(), d),
                 lambda: gmb.dropout(x.cpu(), d), lambda: gmb.dropout(x, 0.5), lambda: gmb.dropout(x.t(), d),
                 lambda: gmb.dropout(x[:1].expand(4, 8), d), lambda: gmb.dropout(x, d, residual=x[:2]),
                 lambda: gmb.dropout(x, d, residual=x.bfloat16()), lambda: gmb.dropout(x, d, ids=torch.zeros(4, device="cuda")),
                 lambda: gmb.dropout(x, d, ids=torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: gmb.rms_norm(x, g[:4]), lambda: gmb.rms_norm(x, g.double()), lambda: gmb.rms_norm(x, g, 0.0),
                 lambda: gmb.rms_norm(x, g, bits=6), lambda: gmb.rms_norm(x, g, out=torch.empty(4, 9, device="cuda")),
                 lambda: gmb.rms_norm(x, g, residual=x, sum_out=x, out=x),
                 lambda: gmb.rms_norm_backward(x, x.bfloat16(), g), lambda: gmb.rms_norm_backward(x[:2], x, g)]:
        with pytest.raises((TypeError, ValueError, gmb.GmbError)):
            call()


def test_more_rows_than_a_grid():
    """Rows past one turn of the grids (65,536 rows of 4 lanes by 16 workgroups a CU and more)."""
    n, dim = 300_001, 9
    x, g = rows(n, dim, 21, torch.float32), torch.rand(dim, device="cuda")
    d = gmb.Dropout(0.5, 8)
    y = gmb.dropout(x, d)
    at = [0, 1, 65535, 262143, 262144, n - 1]
    kept = head_ref.keep(at, dim, 0.5, 8)
    assert torch.equal(y[at].cpu(), torch.where(kept, x[at].cpu() * 2, torch.zeros(())))
    norm, _ = gmb.rms_norm(x, g, EPS)
    want = head_ref.rms_norm(wide(x), wide(g), EPS)
    near(norm, want, 64 * U32 * want.abs(), "norm")
    got = gmb.rms_norm_backward(x, x, g, EPS)
    dr, dw = head_ref.rms_norm_backward(wide(x), wide(x), wide(g), EPS)
    s = 1 / torch.sqrt(wide(x).square().mean(1, keepdim=True) + EPS)
    # 58 U a term, a chain of at most 5 rows a thread (300,001 over 1,024 workgroups of 64), 64 rows and 128 parts
    near(got.weight, dw, 256 * U32 * (wide(x) ** 2 * s).sum(0), "weight")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_offsets_past_32_bits(dtype):
    """Rows 2^31 + 8 elements apart: the same bits as side by side."""
    n, dim, apart = 3, 300, (1 << 31) + 8
    x, res, g = rows(n, dim, 30, dtype), rows(n, dim, 31, dtype), torch.rand(dim, device="cuda")
    memory = torch.empty((n - 1) * apart + 2 * dim, dtype=dtype, device="cuda")
    far, out = memory.as_strided((n, dim), (apart, 1)), memory.as_strided((n, dim), (apart, 1), dim)
    far.copy_(x)
    d = gmb.Dropout(0.5, 8)
    assert torch.equal(gmb.dropout(far, d, residual=res, out=out), gmb.dropout(x, d, residual=res))
    y, r = gmb.rms_norm(far, g, EPS, residual=res, dropout=d, sum_out=out)
    y2, r2 = gmb.rms_norm(x, g, EPS, residual=res, dropout=d)
    assert torch.equal(y, y2) and torch.equal(r, r2)
    got, want = gmb.rms_norm_backward(far, r, g, EPS, carry=far), gmb.rms_norm_backward(x, r2, g, EPS, carry=x)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_replayed():
    x, res, g = (rows(500, 256, 22 + i, torch.float32) for i in range(3))
    w = g[0].abs().contiguous()
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = gmb.Dropout(0.5, 31, 2, step=step)
    out, total = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(gmb.lib().gmb_rms_norm_workspace_bytes(500, 256), dtype=torch.uint8, device="cuda")

    def work():
        gmb.rms_norm(x, w, EPS, residual=res, dropout=d, out=out, sum_out=total)
        return gmb.rms_norm_backward(g, total, w, EPS, carry=res, dropout=d, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = work()
    for k in (3, 4, 4, 9):
        step.fill_(k)
        x.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in (out, total, grads.x, grads.residual, grads.weight)]
        fresh = work()
        assert all(torch.equal(a, b) for a, b in zip(have, (out, total, fresh.x, fresh.residual, fresh.weight))), k
