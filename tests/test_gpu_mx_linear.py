"""The product of microscaled 4-bit rows and weights on the GPU against 64-bit
sums of what the records stand for.  Products of 4-bit elements are exact in
fp32; a sum of t terms in any order is off by at most t half-steps of the sum
of magnitudes, the bias adds one, bf16 one of its own."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import mx_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402

U32, UBF16 = 2.0 ** -24, 2.0 ** -8


def records(n, dim, rng, spread=6):
    x = (rng.normal(size=(n, dim)) * np.exp2(rng.integers(-spread, spread + 1, size=(n, 1)))).astype(np.float32)
    rec = mx_ref.quantise(x, 4)
    return torch.from_numpy(rec).cuda(), mx_ref.values(rec, dim, 4)


def check(got, pairs, bias, relu, dtype):
    """pairs: (rows, weights) in 64 bits."""
    y = sum(a @ w.T for a, w in pairs)
    mag = sum(np.abs(a) @ np.abs(w).T for a, w in pairs)
    terms = sum(a.shape[1] for a, _ in pairs)
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    tol = (terms + 2) * U32 * mag
    if relu:
        y = np.maximum(y, 0)
    if dtype == torch.bfloat16:
        tol = tol + UBF16 * (np.abs(y) + tol)
    got = got.double().cpu().numpy()
    assert got.shape == y.shape
    off = np.abs(got - y) - tol
    assert np.all(off <= 0), (off.max(), np.unravel_index(off.argmax(), off.shape))


# one kernel after the other, each at odd sizes and where it takes over
SHAPES = [(1, 1, 1), (1, 256, 47), (3, 33, 5), (16, 128, 16), (17, 100, 33), (64, 64, 64), (65, 129, 65),
          (100, 515, 130), (33, 4096, 70), (300, 16, 8), (1, 4096, 1030), (257, 384, 256), (1000, 75, 41),
          (2, 65536, 3), (300, 2000, 90), (500, 512, 128), (64, 600, 33),              # few rows
          (20, 40, 9000), (4500, 100, 256), (9000, 300, 129), (70000, 33, 17), (17000, 700, 60), (3000, 1030, 520),
          (3000, 1030, 2100), (8200, 600, 800), (25000, 500, 250),                     # tiles of 64 and 128
          (16500, 530, 600), (2000, 1500, 6200), (66000, 270, 130),                    # tiles of 256
          (120000, 33, 17), (115000, 250, 64), (60000, 100, 100), (58000, 33, 65), (30000, 100, 256),
          (9700, 200, 700)]                                                            # resident weights


@pytest.mark.parametrize("n, d_in, d_out", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_one_pair(n, d_in, d_out, dtype):
    print(f"{n} x {d_in} x {d_out} {dtype}", flush=True)
    rng = np.random.default_rng(n + d_in)
    a, av = records(n, d_in, rng)
    w, wv = records(d_out, d_in, rng)
    check(gmb.mx_linear(a, w, d_in, dtype=dtype), [(av, wv)], None, False, dtype)


@pytest.mark.parametrize("n, d_in, d_out", [s for s in SHAPES if s[1] <= 4096 and s[0] * s[1] * s[2] < 4e9])
@pytest.mark.parametrize("by_id", [False, True])
def test_two_pairs_bias_relu(n, d_in, d_out, by_id):
    print(f"{n} x {d_in} x {d_out}, by id {by_id}", flush=True)
    rng = np.random.default_rng(d_out + d_in)
    store = 50 if by_id else n
    a, av = records(store, d_in, rng)
    a2, a2v = records(n, d_in, rng)
    w, wv = records(d_out, d_in, rng)
    w2, w2v = records(d_out, d_in, rng)
    bias = rng.normal(size=d_out).astype(np.float32)
    ids = None
    if by_id:
        at = rng.integers(0, store, size=n).astype(np.int32)
        ids, av = torch.from_numpy(at).cuda(), av[at]
    for dtype in (torch.float32, torch.bfloat16):
        got = gmb.mx_linear(a, w, d_in, bias=torch.from_numpy(bias).cuda(), a2=a2, w2=w2, ids=ids, relu=True,
                            dtype=dtype)
        check(got, [(av, wv), (a2v, w2v)], bias.astype(np.float64), True, dtype)


@pytest.mark.parametrize("d_in, d_out", [(2100, 60), (2100, 128), (2100, 130), (40, 64), (40, 127), (40, 255)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_large_results(d_in, d_out, dtype):
    """Results past 16 MB, from 50 rows by id, in tiles of every size and with
    resident weights; what lies behind them stays."""
    n = (1 << 24) // (d_out * (4 if dtype == torch.float32 else 2)) + 77
    print(f"{n} x {d_in} x {d_out} {dtype}", flush=True)
    rng = np.random.default_rng(d_in + d_out)
    a, av = records(50, d_in, rng)
    w, wv = records(d_out, d_in, rng, 1)
    ids = rng.integers(0, 50, size=n).astype(np.int32)
    out = torch.full((n + 3, d_out), 7.0, dtype=dtype, device="cuda")
    gmb.mx_linear(a, w, d_in, ids=torch.from_numpy(ids).cuda(), dtype=dtype, out=out)
    assert bool((out[n:] == 7).all())
    y, mag = av @ wv.T, np.abs(av) @ np.abs(wv).T
    tol = (d_in + 2) * U32 * mag
    if dtype == torch.bfloat16:
        tol = tol + UBF16 * (np.abs(y) + tol)
    got = out[:n].double()
    at = torch.from_numpy(ids).cuda().long()
    assert bool(((got - torch.from_numpy(y).cuda()[at]).abs() <= torch.from_numpy(tol).cuda()[at]).all())


@pytest.mark.parametrize("n, d_in, d_out", [(12_300, 2100, 1024), (52_600, 2100, 160), (26_400, 2100, 160),
                                            (264_000, 40, 64), (87_500, 40, 96), (65_700, 40, 128), (33_000, 40, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_large_results_of_whole_pieces(n, d_in, d_out, dtype):
    """Results past 16 MB whose rows are whole 64-byte pieces (those are stored
    past the caches): in tiles of 256 and 128 and with resident weights of each
    shape, from 50 rows by id; what lies behind them stays."""
    print(f"{n} x {d_in} x {d_out} {dtype}", flush=True)
    rng = np.random.default_rng(n)
    a, av = records(50, d_in, rng)
    w, wv = records(d_out, d_in, rng, 1)
    ids = rng.integers(0, 50, size=n).astype(np.int32)
    out = torch.full((n + 3, d_out), 7.0, dtype=dtype, device="cuda")
    gmb.mx_linear(a, w, d_in, ids=torch.from_numpy(ids).cuda(), dtype=dtype, out=out)
    assert bool((out[n:] == 7).all())
    y, mag = av @ wv.T, np.abs(av) @ np.abs(wv).T
    tol = (d_in + 2) * U32 * mag
    if dtype == torch.bfloat16:
        tol = tol + UBF16 * (np.abs(y) + tol)
    at = torch.from_numpy(ids).cuda().long()
    off = (out[:n].double() - torch.from_numpy(y).cuda()[at]).abs() - torch.from_numpy(tol).cuda()[at]
    assert float(off.max()) <= 0


def test_padded_strides_and_given_output():
    rng = np.random.default_rng(8)
    a, av = records(70, 100, rng)
    w, wv = records(30, 100, rng)
    wide = torch.full((70, 160), 0xFF, dtype=torch.uint8, device="cuda")
    wide[:, :80] = a
    wide_w = torch.full((30, 96), 0xFF, dtype=torch.uint8, device="cuda")
    wide_w[:, :80] = w
    out = torch.full((75, 30), 9.0, device="cuda")
    got = gmb.mx_linear(wide, wide_w, 100, out=out)
    assert got is out and bool((out[70:] == 9).all())
    check(out[:70], [(av, wv)], None, False, torch.float32)


def test_what_is_no_number():
    """A block of scale 255 makes its row's (or its column's) results NaN and
    no others; after the activation NaN is 0, as in the other layers."""
    rng = np.random.default_rng(4)
    a, av = records(20, 96, rng)
    w, wv = records(40, 96, rng)
    a[3, 48 + 1] = 255
    w[7, 48 + 2] = 255
    y = gmb.mx_linear(a, w, 96).cpu().numpy()
    bad = np.zeros((20, 40), bool)
    bad[3] = True
    bad[:, 7] = True
    assert np.array_equal(np.isnan(y), bad)
    assert np.array_equal(gmb.mx_linear(a, w, 96, relu=True).cpu().numpy()[bad], np.zeros(bad.sum(), np.float32))


def test_ids_outside_count_as_zeros(dg):
    from gpu_util import csr_on_device
    csr = csr_on_device(dg.rmat(8, 200, 900, (0.57, 0.19, 0.19), 4))
    rng = np.random.default_rng(4)
    a, av = records(20, 64, rng)
    a2, a2v = records(6, 64, rng)
    w, wv = records(40, 64, rng)
    a[0, 32:34] = 255                          # record 0 must not leak into rows without a record
    ids = torch.tensor([5, -1, 19, 20, 7, 1 << 30], dtype=torch.int32, device="cuda")
    y = gmb.mx_linear(a, w, 64, a2=a2, w2=w, ids=ids, status_word=csr.status_word)
    rows = np.zeros((6, 64))
    rows[[0, 2, 4]] = av[[5, 19, 7]]
    check(y, [(rows, wv), (a2v, wv)], None, False, torch.float32)
    with pytest.raises(gmb.GmbError, match="ERANGE"):
        csr.check_status()


def test_scales_far_apart():
    """Blocks whose scales differ by 2^60: small terms next to large ones."""
    rng = np.random.default_rng(6)
    x = (rng.normal(size=(40, 256)) * np.exp2(rng.integers(-30, 31, size=(40, 8))).repeat(32, 1)).astype(np.float32)
    v = (rng.normal(size=(50, 256)) * np.exp2(rng.integers(-30, 31, size=(50, 8))).repeat(32, 1)).astype(np.float32)
    a, w = mx_ref.quantise(x, 4), mx_ref.quantise(v, 4)
    got = gmb.mx_linear(torch.from_numpy(a).cuda(), torch.from_numpy(w).cuda(), 256)
    check(got, [(mx_ref.values(a, 256, 4), mx_ref.values(w, 256, 4))], None, False, torch.float32)


def test_a_graph_replayed():
    rng = np.random.default_rng(1)
    a, _ = records(500, 200, rng)
    w, wv = records(90, 200, rng)
    out = torch.empty((500, 90), device="cuda")
    gmb.mx_linear(a, w, 200, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gmb.mx_linear(a, w, 200, out=out)
    for _ in range(3):
        b, bv = records(500, 200, rng)
        a.copy_(b)
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(out, [(bv, wv)], None, False, torch.float32)


def test_refusals():
    rng = np.random.default_rng(1)
    a, _ = records(5, 64, rng)
    w, _ = records(7, 64, rng)
    ids = torch.zeros(5, dtype=torch.int32, device="cuda")
    bias = torch.zeros(7, device="cuda")
    for call in (lambda: gmb.mx_linear(a, w, 65), lambda: gmb.mx_linear(a, w, 0), lambda: gmb.mx_linear(a.int(), w, 64),
                 lambda: gmb.mx_linear(a, w, 64, a2=a), lambda: gmb.mx_linear(a, w, 64, a2=a[:4], w2=w),
                 lambda: gmb.mx_linear(a, w, 64, a2=a, w2=w[:6]), lambda: gmb.mx_linear(a, w, 64, bias=bias[:6]),
                 lambda: gmb.mx_linear(a, w, 64, bias=bias.double()), lambda: gmb.mx_linear(a, w, 64, ids=ids.long()),
                 lambda: gmb.mx_linear(a, w, 64, dtype=torch.float16),
                 lambda: gmb.mx_linear(a, w, 64, out=torch.empty(5, 6, device="cuda"))):
        with pytest.raises((TypeError, ValueError, gmb.GmbError)):
            call()
    assert gmb.mx_linear(a, w, 64, ids=ids[:0]).shape == (0, 7)
