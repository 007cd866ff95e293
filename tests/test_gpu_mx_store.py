"""The microscaled store on the GPU: rows written into it and read back bit
for bit, and its mean, against the numpy definitions."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import mx_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402
from gpu_util import csr_on_device  # noqa: E402

U32, UBF16 = 2.0 ** -24, 2.0 ** -8
DTYPES = [torch.float32, torch.bfloat16]


def rows_of(n, dim, seed, dtype=torch.float32):
    """Rows of normal values over many binades, with rows of zeros, of
    denormals, of the largest values, and blocks that hold an infinity or NaN."""
    rng = np.random.default_rng(seed)
    x = (rng.normal(size=(n, dim)) * np.exp2(rng.integers(-20, 20, size=(n, 1)))).astype(np.float32)
    special = [0.0, -0.0, 2.0 ** -140, 3.0e38, np.inf, np.nan, 2.0 ** -126, -2.0 ** -127]
    for i, s in enumerate(special):
        if i + 2 < n:
            if np.isfinite(s):
                x[i + 2] = s * np.where(rng.random(dim) < 0.5, 1, 0.3)
            else:
                x[i + 2, dim // 2] = s
    t = torch.from_numpy(x).to(dtype)
    return t.cuda(), t.float().numpy()


def same(a, b):
    return np.array_equal(np.asarray(a), np.asarray(b), equal_nan=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("n, dim", [(1, 1), (7, 16), (13, 31), (64, 32), (65, 33), (40, 75), (33, 100), (300, 128),
                                    (17, 161), (9, 256), (21, 515), (5, 1024), (3, 4096), (2, 65536)])
def test_write_and_read(n, dim, bits, dtype):
    print(f"{n} rows of {dim}, {bits} bits, {dtype}", flush=True)
    x, host = rows_of(n, dim, 100 * dim + n, dtype)
    rec = gmb.mx_quantise(x, bits)
    want = mx_ref.quantise(host, bits)
    assert np.array_equal(rec.cpu().numpy(), want)
    v = mx_ref.values(want, dim, bits)
    assert same(gmb.mx_gather(None, rec, dim, bits).cpu().numpy(), v.astype(np.float32))
    got = gmb.mx_gather(None, rec, dim, bits, dtype=torch.bfloat16)
    assert same(got.float().cpu().numpy(), mx_ref.bf16(v.astype(np.float32)))


@pytest.mark.parametrize("bits", [4, 8])
def test_every_rounding_and_tie(bits):
    """Every value between two neighbouring elements' quarters, at three
    scales, both signs; the first element of a block fixes its scale."""
    grid = mx_ref.FP4 if bits == 4 else mx_ref.FP8
    q = np.unique(np.concatenate([grid[:-1] + f * np.diff(grid) for f in (0, .25, .5, .75, .49999, .50001)]))
    q = np.concatenate([q, -q, [grid[-1] * 1.3, -grid[-1] * 1.3]])
    rows = []
    for e in (-100, 0, 90):
        for at in range(0, len(q), 31):
            r = np.zeros(32)
            r[0] = grid[-1]                                 # the block's scale is 2^e
            part = q[at:at + 31]
            r[1:1 + len(part)] = part
            rows.append(np.ldexp(r, e))
    x = np.array(rows, np.float32)
    rec = gmb.mx_quantise(torch.from_numpy(x).cuda(), bits).cpu().numpy()
    assert np.array_equal(rec, mx_ref.quantise(x, bits))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("d_in, d_out", [(1, 1), (16, 8), (75, 41), (100, 256), (256, 47), (515, 130), (4096, 5)])
def test_columns_of_a_matrix(d_in, d_out, bits, dtype):
    w, host = rows_of(d_in, d_out, d_in, dtype)
    rec = gmb.mx_quantise(w.t(), bits)
    assert np.array_equal(rec.cpu().numpy(), mx_ref.quantise(host.T, bits))


def test_strided_rows():
    """Rows and columns at a stride, one row for all, rows at odd addresses."""
    rng = np.random.default_rng(5)
    host = rng.normal(size=(40, 90)).astype(np.float32)
    big = torch.from_numpy(host).cuda()
    for view, want in [(big[::3, 1:76], host[::3, 1:76]), (big[:, 5:90:2], host[:, 5:90:2]),
                       (big[4:5].expand(6, 90), host[4:5].repeat(6, 0)), (big[2:3, 7:9], host[2:3, 7:9]),
                       (big[:, 3:4].expand(40, 33), host[:, 3:4].repeat(33, 1))]:
        assert np.array_equal(gmb.mx_quantise(view, 4).cpu().numpy(), mx_ref.quantise(want, 4))
    b16 = big.bfloat16()[:, 1:38]
    assert np.array_equal(gmb.mx_quantise(b16, 8).cpu().numpy(), mx_ref.quantise(b16.float().cpu().numpy(), 8))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [16, 100, 300])
def test_write_by_id(dim, bits):
    """Ids in no order; rows that no id names, and the bytes between a record
    and the next, stay as they were; a padded row stride."""
    rng = np.random.default_rng(dim)
    rows, n = 500, 200
    rec = mx_ref.record_bytes(dim, bits)
    table = torch.full((rows, rec + 48), 0xA5, dtype=torch.uint8, device="cuda")[:, :rec + 16]
    x, host = rows_of(n, dim, 7)
    ids = rng.permutation(rows)[:n].astype(np.int32)
    before = table.cpu().numpy().copy()
    out = gmb.mx_quantise(x, bits, ids=torch.from_numpy(ids).cuda(), table=table)
    assert out is table
    want = before.copy()
    want[ids, :rec] = mx_ref.quantise(host, bits)
    assert np.array_equal(table.cpu().numpy(), want)
    got = gmb.mx_gather(torch.from_numpy(ids).cuda(), table, dim, bits).cpu().numpy()
    assert same(got, mx_ref.values(want[ids, :rec], dim, bits).astype(np.float32))
    first = gmb.mx_gather(torch.from_numpy(ids).cuda(), table, dim, bits, n=3)
    assert first.shape == (3, dim) and same(first.cpu().numpy(), got[:3])


@pytest.fixture(scope="module")
def graph(dg):
    g = dg.rmat(13, 6_000, 40_000, (0.57, 0.19, 0.19), 4)
    return g, csr_on_device(g)


@pytest.mark.parametrize("turned", [False, True])
def test_the_last_row_of_an_id_counts(graph, turned):
    """With a graph's sampler state an id may come often; the state is clear
    again afterwards (the sampler's own results are as before)."""
    g, csr = graph
    rng = np.random.default_rng(2)
    n, dim = 5000, 70
    ids = rng.integers(0, 300, size=n).astype(np.int32) * 19
    ids[-1] = ids[0]
    host = rng.normal(size=(n, dim)).astype(np.float32)
    x = torch.from_numpy(host.T.copy()).cuda().t() if turned else torch.from_numpy(host).cuda()
    table = torch.zeros((g.num_nodes, mx_ref.record_bytes(dim, 4)), dtype=torch.uint8, device="cuda")
    seeds = torch.arange(100, dtype=torch.int32, device="cuda")
    before = [b.src_ids.clone() for b in gmb.sample_blocks(csr, seeds, [5, 5], 3).blocks()]
    gmb.mx_quantise(x, 4, ids=torch.from_numpy(ids).cuda(), table=table, csr=csr)
    want = np.zeros(table.shape, np.uint8)
    want[ids] = mx_ref.quantise(host, 4)      # numpy: the last one stays
    last = {int(v): i for i, v in enumerate(ids)}
    assert np.array_equal(want[list(last)], mx_ref.quantise(host, 4)[list(last.values())])
    assert np.array_equal(table.cpu().numpy(), want)
    csr.check_status()
    after = [b.src_ids for b in gmb.sample_blocks(csr, seeds, [5, 5], 3).blocks()]
    assert all(torch.equal(a, b) for a, b in zip(before, after))


def test_ids_outside_the_table(graph):
    g, csr = graph
    x = torch.ones(4, 32, device="cuda")
    table = torch.zeros((g.num_nodes, 32), dtype=torch.uint8, device="cuda")
    ids = torch.tensor([3, -1, g.num_nodes, 5], dtype=torch.int32, device="cuda")
    for state in (None, csr):
        table.zero_()
        gmb.mx_quantise(x, 4, ids=ids, table=table, csr=state, status_word=csr.status_word)
        assert sorted(torch.nonzero(table.any(1))[:, 0].tolist()) == [3, 5]
        with pytest.raises(gmb.GmbError, match="ERANGE"):
            csr.check_status()
    got = gmb.mx_gather(ids, table, 32, 4, status_word=csr.status_word)
    assert got[:, 0].tolist() == [1.0, 0.0, 0.0, 1.0]
    with pytest.raises(gmb.GmbError, match="ERANGE"):
        csr.check_status()
    csr.check_status()


def test_a_sampled_batch(graph):
    """Blocks in place of ids: the input vertices, their number on the device;
    rows past it stay as they were."""
    g, csr = graph
    dim = 60
    rng = np.random.default_rng(9)
    feats = rng.normal(size=(g.num_nodes, dim)).astype(np.float32)
    table = gmb.mx_quantise(torch.from_numpy(feats).cuda(), 8)
    blocks = gmb.sample_blocks(csr, torch.arange(50, dtype=torch.int32, device="cuda"), [7, 4], 1)
    n_src, cap = blocks.sizes()[0][1], blocks.input_capacity
    out = torch.full((cap, dim), 7.0, device="cuda")
    got = gmb.mx_gather(blocks, table, dim, 8, out=out)
    ids = blocks.input_ids[:n_src].cpu().numpy()
    v = mx_ref.values(mx_ref.quantise(feats, 8), dim, 8)
    assert same(got[:n_src].cpu().numpy(), v[ids].astype(np.float32)) and bool((got[n_src:] == 7).all())
    x = torch.full((cap, dim), 2.0, device="cuda")
    before = table.cpu().numpy()
    gmb.mx_quantise(x, 8, ids=blocks, table=table)
    want = before.copy()
    want[ids] = mx_ref.quantise(np.full((1, dim), 2.0), 8)
    assert np.array_equal(table.cpu().numpy(), want)
    m = gmb.mx_mean(blocks, table, dim, 8)
    b = blocks.blocks()[0]
    ref, mag = mx_ref.mean(b.indptr.cpu().numpy(), b.nbr.cpu().numpy(), mx_ref.values(want, dim, 8))
    assert np.all(np.abs(m[:b.n_dst].cpu().numpy() - ref) <= (7 + 2) * U32 * mag)
    csr.check_status()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("n, most, dim", [(1, 1, 1), (64, 5, 16), (3, 0, 40), (50, 40, 75), (33, 17, 100),
                                          (20, 9, 128), (70, 33, 200), (9, 16, 515), (5, 300, 64), (2, 3, 4100)])
def test_mean(n, most, dim, bits, dtype):
    """Destinations without and with many neighbours.  fp32 sums of k terms
    and a division: (k + 1) half-steps of the mean magnitude; bf16 one more
    rounding."""
    rng = np.random.default_rng(n + dim)
    store = 200
    x = (rng.normal(size=(store, dim)) * np.exp2(rng.integers(-6, 6, size=(store, 1)))).astype(np.float32)
    rec = mx_ref.quantise(x, bits)
    k = rng.integers(0, most + 1, size=n)
    if n > 2:
        k[0], k[-1] = most, 0
    indptr = np.concatenate([[0], np.cumsum(k)]).astype(np.int32)
    ids = rng.integers(0, store, size=indptr[-1]).astype(np.int32)
    got = gmb.mx_mean((torch.from_numpy(indptr).cuda(), torch.from_numpy(ids).cuda()), torch.from_numpy(rec).cuda(),
                      dim, bits, dtype=dtype)
    ref, mag = mx_ref.mean(indptr, ids, mx_ref.values(rec, dim, bits))
    tol = (k[:, None] + 2) * U32 * mag + (UBF16 * np.abs(ref) if dtype == torch.bfloat16 else 0)
    assert got.shape == (n, dim) and got.dtype == dtype
    assert np.all(np.abs(got.double().cpu().numpy() - ref) <= tol)


def test_mean_of_what_is_no_number():
    """A block of scale 255 spreads to its own 32 elements, and only to the
    destinations that have it; ids outside the store are record 0."""
    x = np.ones((4, 64), np.float32)
    x[1, 3] = np.nan
    x[2] = 3.0
    rec = torch.from_numpy(mx_ref.quantise(x, 4)).cuda()
    indptr = torch.tensor([0, 2, 4, 4, 6], dtype=torch.int32, device="cuda")
    ids = torch.tensor([0, 1, 2, 3, -5, 400], dtype=torch.int32, device="cuda")
    m = gmb.mx_mean((indptr, ids), rec, 64, 4).cpu().numpy()
    assert np.isnan(m[0, :32]).all() and np.all(m[0, 32:] == 1)
    assert np.all(m[1] == 2) and np.all(m[2] == 0) and np.all(m[3] == 1)


def test_addresses_past_32_bits():
    """A store of 6 GB: its last rows written, read and averaged."""
    dim, rows = 128, 75_000_000
    table = torch.empty((rows, mx_ref.record_bytes(dim, 4)), dtype=torch.uint8, device="cuda")
    x, host = rows_of(64, dim, 3)
    host[:, :] = np.where(np.isfinite(host), host, 1.0)
    x = torch.from_numpy(host).cuda()
    at = np.linspace(1, rows - 1, 64).astype(np.int32)
    ids = torch.from_numpy(at).cuda()
    print("write, read, mean at rows up to", at[-1], flush=True)
    gmb.mx_quantise(x, 4, ids=ids, table=table)
    v = mx_ref.values(mx_ref.quantise(host, 4), dim, 4)
    assert same(gmb.mx_gather(ids, table, dim, 4).cpu().numpy(), v.astype(np.float32))
    indptr = torch.arange(65, dtype=torch.int32, device="cuda")
    assert same(gmb.mx_mean((indptr, ids), table, dim, 4).cpu().numpy(), v.astype(np.float32))
    w = torch.from_numpy(mx_ref.quantise(np.eye(128, dtype=np.float32), 4)).cuda()
    assert same(gmb.mx_linear(table, w, dim, ids=ids).cpu().numpy(), v.astype(np.float32))


@pytest.mark.parametrize("dim", [75, 500])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_large_results(dim, dtype):
    """Reads and means past 16 MB, of 60 records; what lies behind them stays."""
    size = 4 if dtype == torch.float32 else 2
    n = (1 << 24) // (dim * size) + 5
    print(f"{n} rows of {dim} {dtype}", flush=True)
    rng = np.random.default_rng(dim)
    rec = mx_ref.quantise(rng.normal(size=(60, dim)).astype(np.float32), 8)
    table, val = torch.from_numpy(rec).cuda(), torch.from_numpy(mx_ref.values(rec, dim, 8)).cuda()
    ids = torch.from_numpy(rng.integers(0, 60, size=2 * n).astype(np.int32)).cuda()
    out = torch.full((n + 3, dim), 7.0, dtype=dtype, device="cuda")
    gmb.mx_gather(ids, table, dim, 8, dtype=dtype, n=n, out=out)
    assert bool((out[n:] == 7).all())
    # (values of 8 bits: exact in bf16)
    assert torch.equal(out[:n].double(), val[ids[:n].long()])
    indptr = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda")
    out.fill_(7)
    gmb.mx_mean((indptr, ids), table, dim, 8, dtype=dtype, out=out)
    assert bool((out[n:] == 7).all())
    pair = val[ids.long()].view(n, 2, dim)
    # the sum of two values of 8 bits rounds once (fp32), half of it never, bf16 once more
    tol = 2.0 ** -24 * pair.abs().sum(1) + (2.0 ** -8 * pair.sum(1).abs() if size == 2 else 0)
    assert bool(((out[:n].double() - pair.mean(1)).abs() <= tol).all())


def test_a_mean_of_more_rows_than_a_grid_counts():
    """2^26 + 9 rows of 64 lanes are more threads than 32 bits count."""
    n, dim = (1 << 26) + 9, 257
    print(f"mean: {n} rows of {dim}", flush=True)
    x = torch.from_numpy(np.random.default_rng(1).normal(size=(9, dim)).astype(np.float32)).cuda()
    table = gmb.mx_quantise(x, 4)
    indptr = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    indptr[-9:] = torch.arange(1, 10, dtype=torch.int32, device="cuda")
    out = torch.empty((n, dim), dtype=torch.bfloat16, device="cuda")
    out[:: 4097] = float("nan")
    out[-9:] = float("nan")
    ids = torch.arange(8, -1, -1, dtype=torch.int32, device="cuda")
    gmb.mx_mean((indptr, ids), table, dim, 4, dtype=torch.bfloat16, out=out)
    want = gmb.mx_gather(ids, table, dim, 4, dtype=torch.bfloat16)
    assert torch.equal(out[-9:], want)
    assert bool((out[:-9][:: 4097] == 0).all())
    del out
    torch.cuda.empty_cache()


def test_another_stream_and_a_graph():
    """Work on a stream of its own, and captured and replayed with other rows
    in the same buffers."""
    dim, n, rows = 90, 700, 4000
    x, host = rows_of(n, dim, 1)
    rng = np.random.default_rng(0)
    ids = torch.from_numpy(rng.permutation(rows)[:n].astype(np.int32)).cuda()
    indptr = torch.arange(0, n + 1, 10, dtype=torch.int32, device="cuda")
    table = torch.zeros((rows, mx_ref.record_bytes(dim, 4)), dtype=torch.uint8, device="cuda")
    back = torch.empty((n, dim), device="cuda")
    avg = torch.empty((n // 10, dim), device="cuda")

    def work():
        gmb.mx_quantise(x, 4, ids=ids, table=table)
        gmb.mx_gather(ids, table, dim, 4, out=back)
        gmb.mx_mean((indptr, ids), table, dim, 4, out=avg)

    def check(host):
        v = mx_ref.values(mx_ref.quantise(host, 4), dim, 4)
        assert same(back.cpu().numpy(), v.astype(np.float32))
        ref, mag = v.reshape(-1, 10, dim).mean(1), np.abs(v).reshape(-1, 10, dim).mean(1)
        ok = np.isnan(ref) & np.isnan(avg.cpu().numpy()) | (np.abs(avg.cpu().numpy() - ref) <= 12 * U32 * mag)
        assert ok.all()

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work()
    s.synchronize()
    check(host)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work()
    for seed in (5, 6, 7):
        y, host = rows_of(n, dim, seed)
        x.copy_(y)
        back.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(host)


def test_refusals(graph):
    g, csr = graph
    x = torch.zeros(4, 40, device="cuda")
    rec = gmb.mx_quantise(x, 4)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [lambda: gmb.mx_quantise(x.half(), 4), lambda: gmb.mx_quantise(x[0], 4), lambda: gmb.mx_quantise(x, 5),
           lambda: gmb.mx_quantise(x, 4, ids=ids), lambda: gmb.mx_quantise(x, 4, ids=ids[:3], table=rec),
           lambda: gmb.mx_quantise(x, 4, table=rec[:3]), lambda: gmb.mx_quantise(x, 8, table=rec),
           lambda: gmb.mx_quantise(x, 4, ids=ids.long(), table=rec),
           lambda: gmb.mx_quantise(x, 4, ids=ids, table=rec, csr=csr),
           lambda: gmb.mx_quantise(x, 4, table=rec.float()), lambda: gmb.mx_quantise(x, 4, table=rec[:, 1:]),
           lambda: gmb.mx_gather(ids, rec, 40, 8), lambda: gmb.mx_gather(ids, rec, 400, 4),
           lambda: gmb.mx_gather(ids, rec, 40, 4, n=5), lambda: gmb.mx_gather(None, rec, 40, 4, n=5),
           lambda: gmb.mx_gather(ids, rec, 40, 4, dtype=torch.float16),
           lambda: gmb.mx_gather(ids, rec, 40, 4, out=torch.empty(3, 40, device="cuda")),
           lambda: gmb.mx_gather(ids, rec, 0, 4), lambda: gmb.mx_mean((ids, ids.cpu()), rec, 40, 4),
           lambda: gmb.mx_mean((ids.view(2, 2), ids), rec, 40, 4),
           lambda: gmb.mx_mean((ids, ids), rec, 40, 4, out=torch.empty(3, 39, device="cuda"))]
    for call in bad:
        with pytest.raises((TypeError, ValueError, gmb.GmbError)):
            call()
    empty = gmb.mx_quantise(x[:0], 4)
    assert empty.shape == (0, rec.shape[1]) and gmb.mx_gather(None, empty, 40, 4).shape == (0, 40)
    assert gmb.mx_gather(ids[:0], rec, 40, 4).shape == (0, 40)
    assert gmb.mx_mean((ids[:1], ids[:0]), rec, 40, 4).shape == (0, 40)
