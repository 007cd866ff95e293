"""The microscaled operators and the distillation loss as they are used: a
model and a store in 4 bits served by sage_forward_mx, a student trained from
a teacher's top logits through sage_backward, and both together."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import mx_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402
from gpu_util import csr_on_device, to_torch_weights  # noqa: E402

U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def graph(dg):
    g = dg.rmat(14, 12_000, 120_000, (0.57, 0.19, 0.19), 11)
    return g, csr_on_device(g)


# ---------------------------------------------------------------- serving

def check_records(rec, y, tol, what):
    """Records of quantised values that are within `tol` of y: the scale is
    that of a largest magnitude within tol of y's, and every element is as
    near to y as its scale allows, up to 2 tol."""
    n, dim = y.shape
    nb = (dim + 31) // 32
    codes = rec[:, nb * 16:nb * 17].astype(np.int64)
    pad = lambda a: np.pad(a, ((0, 0), (0, nb * 32 - dim))).reshape(n, nb, 32)  # noqa: E731
    yb, tb = pad(np.abs(y)), pad(tol)
    lo = mx_ref.scale_code(np.maximum(yb - tb, 0).max(2).astype(np.float32) * np.float32(1 - 2 * U32), 4)
    hi = mx_ref.scale_code((yb + tb).max(2).astype(np.float32) * np.float32(1 + 2 * U32), 4)
    assert np.all((lo <= codes) & (codes <= hi)), what
    s = mx_ref.scale_of(codes)[:, :, None]
    m = yb / s
    apart = np.abs(m - mx_ref.FP4[mx_ref.nearest(m, mx_ref.FP4)]) * s
    v = pad(mx_ref.values(rec, dim, 4))
    assert np.all(np.abs(v - pad(y)) <= apart + 2 * tb), what
    raw = rec[:, :nb * 16].reshape(n, nb, 16)
    raw = np.stack((raw & 7, (raw >> 4) & 7), 3).reshape(n, nb * 32)
    assert np.all(raw[:, dim:] == 0) and np.all(rec[:, nb * 17:] == 0), what


def served(blocks, table, weights, mxw):
    """sage_forward_mx, every layer against 64-bit sums of the records that it
    read itself."""
    need = gmb.mx_forward_workspace_bytes(blocks, mxw)
    ws = gmb._aligned_bytes(need, table.device)[1]
    ws.fill_(0xAA)
    logits = gmb.sage_forward_mx(blocks, table, mxw, workspace=ws)
    blocks.csr.check_status()
    L, dims = blocks.num_layers, mxw.dims
    whole = ws.cpu().numpy()
    host = blocks.blocks()
    src = host[0].src_ids.cpu().numpy()
    stored = table.cpu().numpy()[:, :mx_ref.record_bytes(dims[0], 4)]

    def records(l, hidden):
        off = gmb.lib().gmb_mx_forward_offset(ctypes.byref(blocks.struct), ctypes.byref(mxw.struct), l, hidden)
        rb = mx_ref.record_bytes(dims[l + hidden], 4)
        return whole[off:off + host[l].n_dst * rb].reshape(host[l].n_dst, rb)

    h = mx_ref.values(stored[src], dims[0], 4)              # layer 0's inputs, by position
    for l, b in enumerate(host):
        ref, mag = mx_ref.mean(b.indptr.cpu().numpy(), b.indices.cpu().numpy(), h)
        k = np.diff(b.indptr.cpu().numpy())[:, None]
        check_records(records(l, 0), ref, (k + 2) * U32 * mag, f"layer {l} mean")
        m = mx_ref.values(records(l, 0), dims[l], 4)
        wsf = mx_ref.values(mxw.w_self[l].cpu().numpy(), dims[l], 4)
        wnb = mx_ref.values(mxw.w_neigh[l].cpu().numpy(), dims[l], 4)
        bias = mxw.bias[l].double().cpu().numpy()
        hd = h[:b.n_dst]
        z = hd @ wsf.T + m @ wnb.T + bias
        tol = (2 * dims[l] + 2) * U32 * (np.abs(hd) @ np.abs(wsf).T + np.abs(m) @ np.abs(wnb).T + np.abs(bias))
        if l + 1 < L:
            z = np.maximum(z, 0)
            check_records(records(l, 1), z, tol, f"layer {l} hidden")
            h = mx_ref.values(records(l, 1), dims[l + 1], 4)
        else:
            assert np.all(np.abs(logits.double().cpu().numpy() - z) <= tol), f"layer {l} logits"
    return logits


@pytest.mark.parametrize("dims, fanouts, seeds", [([16, 16, 8], [5, 5], 64), ([100, 256, 47], [10, 5], 300),
                                                  ([75, 100, 64, 41], [6, 4, 3], 33), ([128, 47], [25], 500),
                                                  ([33, 70, 5], [4, 300], 7), ([40, 31, 3], [2, 2], 1)])
def test_serving(dg, graph, dims, fanouts, seeds):
    print(f"{dims}, fan-outs {fanouts}, {seeds} seeds", flush=True)
    g, csr = graph
    w = to_torch_weights(dg.sage_weights(dims, 6))
    mxw = gmb.SageMxWeights(w)
    for l in range(len(dims) - 1):
        assert np.array_equal(mxw.w_self[l].cpu().numpy(), mx_ref.quantise(w.w_self[l].t().cpu().numpy(), 4))
        assert np.array_equal(mxw.w_neigh[l].cpu().numpy(), mx_ref.quantise(w.w_neigh[l].t().cpu().numpy(), 4))
    feats = torch.from_numpy(dg.features(g.num_nodes, dims[0], 5, "f32")).cuda()
    table = gmb.mx_quantise(feats, gmb.MXFP4)
    ids = torch.from_numpy(dg.permutation(g.num_nodes, 7)[:seeds]).cuda()
    blocks = gmb.sample_blocks(csr, ids, fanouts, 8)
    a = served(blocks, table, w, mxw)
    # a store with a padded row stride, another workspace: the same bits
    wide = torch.empty((g.num_nodes, table.shape[1] + 32), dtype=torch.uint8, device="cuda")
    wide[:, :table.shape[1]] = table
    assert torch.equal(gmb.sage_forward_mx(blocks, wide, mxw), a)


@pytest.fixture(scope="module")
def wide_graph(dg):
    g = dg.rmat(17, 100_000, 500_000, (0.57, 0.19, 0.19), 13)
    return g, csr_on_device(g)


@pytest.mark.parametrize("d_in, d_hid", [(100, 256), (100, 100), (100, 60),      # resident weights, each shape
                                         (140, 200), (140, 100), (140, 60)])     # tiles of 256, 128 and 64
def test_serving_many_rows(dg, wide_graph, d_in, d_hid):
    """Hidden records of tens of thousands of destinations; rows of the
    workspace past the last destination stay as they were."""
    g, csr = wide_graph
    dims, seeds = [d_in, d_hid, 8], 24_000
    print(f"{dims}, {seeds} seeds", flush=True)
    mxw = gmb.SageMxWeights(to_torch_weights(dg.sage_weights(dims, 6)))
    table = gmb.mx_quantise(torch.from_numpy(dg.features(g.num_nodes, d_in, 5, "f32")).cuda(), gmb.MXFP4)
    ids = torch.from_numpy(dg.permutation(g.num_nodes, 7)[:seeds]).cuda()
    blocks = gmb.sample_blocks(csr, ids, [3, 2], 8)
    cap = int(blocks.struct.blk[0].cap_dst)
    assert cap == 3 * seeds
    want = served(blocks, table, None, mxw)
    ws = gmb._aligned_bytes(gmb.mx_forward_workspace_bytes(blocks, mxw), table.device)[1]
    ws.fill_(0xAA)
    assert torch.equal(gmb.sage_forward_mx(blocks, table, mxw, workspace=ws), want)
    n = blocks.sizes()[0][0]
    assert n < cap
    for hidden in (0, 1):
        rb = mx_ref.record_bytes(dims[hidden], 4)
        off = gmb.lib().gmb_mx_forward_offset(ctypes.byref(blocks.struct), ctypes.byref(mxw.struct), 0, hidden)
        assert bool((ws[off + n * rb:off + cap * rb] == 0xAA).all())


def test_serving_replayed_and_empty(dg, graph):
    g, csr = graph
    dims = [60, 50, 9]
    mxw = gmb.SageMxWeights(to_torch_weights(dg.sage_weights(dims, 2)))
    table = gmb.mx_quantise(torch.from_numpy(dg.features(g.num_nodes, 60, 5, "f32")).cuda(), 4)
    other = gmb.mx_quantise(torch.from_numpy(dg.features(g.num_nodes, 60, 9, "f32")).cuda(), 4)
    blocks = gmb.sample_blocks(csr, torch.arange(77, dtype=torch.int32, device="cuda"), [5, 4], 3)
    ws = gmb._aligned_bytes(gmb.mx_forward_workspace_bytes(blocks, mxw), table.device)[1]
    logits = gmb.sage_forward_mx(blocks, table, mxw, workspace=ws)
    want = [gmb.sage_forward_mx(blocks, t, mxw) for t in (other, table)]
    torch.cuda.synchronize()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        gmb.sage_forward_mx(blocks, table, mxw, workspace=ws, logits=logits)
    first = table.clone()
    for t, w in ((other, want[0]), (first, want[1]), (other, want[0])):
        table.copy_(t)
        logits.zero_()
        torch.cuda.synchronize()
        cg.replay()
        torch.cuda.synchronize()
        assert torch.equal(logits, w)
    empty = gmb.sample_blocks(csr, torch.empty(0, dtype=torch.int32, device="cuda"), [5, 4], 3)
    assert gmb.sage_forward_mx(empty, table, mxw).shape == (0, 9)
    with pytest.raises((TypeError, ValueError)):
        gmb.sage_forward_mx(blocks, table[:, :32], mxw)
    with pytest.raises(ValueError):
        gmb.sage_forward_mx(blocks, table, mxw, logits=torch.empty(76, 9, device="cuda"))
    with pytest.raises(ValueError):
        mxw.requantise(to_torch_weights(dg.sage_weights([60, 40, 9], 2)))


def test_a_store_smaller_than_the_graph(dg, graph):
    """Ids outside the store: reported, in bounds."""
    g, csr = graph
    mxw = gmb.SageMxWeights(to_torch_weights(dg.sage_weights([60, 9], 2)))
    table = gmb.mx_quantise(torch.randn(100, 60, device="cuda"), 4)
    blocks = gmb.sample_blocks(csr, torch.arange(50, 150, dtype=torch.int32, device="cuda"), [5], 3)
    out = gmb.sage_forward_mx(blocks, table, mxw)
    assert torch.isfinite(out).all()
    with pytest.raises(gmb.GmbError, match="ERANGE"):
        csr.check_status()


def test_other_weights_in_a_served_model(dg, graph):
    """requantise with another set of weights (a checkpoint, an average) takes
    its matrices and its biases, also for a graph captured before, and leaves
    the first set as it was."""
    g, csr = graph
    dims = [60, 50, 9]
    first, second = (to_torch_weights(dg.sage_weights(dims, s)) for s in (2, 3))
    assert all(not torch.equal(a, b) for a, b in zip(first.bias, second.bias))
    kept = [b.clone() for b in first.bias]
    mxw = gmb.SageMxWeights(first)
    table = gmb.mx_quantise(torch.from_numpy(dg.features(g.num_nodes, 60, 5, "f32")).cuda(), 4)
    blocks = gmb.sample_blocks(csr, torch.arange(77, dtype=torch.int32, device="cuda"), [5, 4], 3)
    ws = gmb._aligned_bytes(gmb.mx_forward_workspace_bytes(blocks, mxw), table.device)[1]
    logits = gmb.sage_forward_mx(blocks, table, mxw, workspace=ws)
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        gmb.sage_forward_mx(blocks, table, mxw, workspace=ws, logits=logits)
    for w in (second, first, second):
        want = gmb.sage_forward_mx(blocks, table, gmb.SageMxWeights(w))
        mxw.requantise(w)
        assert torch.equal(gmb.sage_forward_mx(blocks, table, mxw), want)
        logits.zero_()
        torch.cuda.synchronize()
        cg.replay()
        torch.cuda.synchronize()
        assert torch.equal(logits, want)
        assert all(torch.equal(a, b) for a, b in zip(mxw.values().bias, w.bias))
    assert all(torch.equal(a, b) for a, b in zip(first.bias, kept))
    short = to_torch_weights(dg.sage_weights(dims, 2))
    short.bias[1] = short.bias[1][:1]
    for call in (lambda: mxw.requantise(short), lambda: gmb.SageMxWeights(short)):
        with pytest.raises(ValueError):
            call()


def test_neighbours_outside_the_store(dg, graph):
    """Destinations inside the store, some of their sampled neighbours outside:
    reported, and read as record 0."""
    g, csr = graph
    dims, rows = [60, 9], 4000
    mxw = gmb.SageMxWeights(to_torch_weights(dg.sage_weights(dims, 2)))
    feats = torch.from_numpy(dg.features(g.num_nodes, 60, 5, "f32")).cuda()
    whole = gmb.mx_quantise(feats, 4)
    blocks = gmb.sample_blocks(csr, torch.arange(0, rows, 7, dtype=torch.int32, device="cuda"), [6], 3)
    b = blocks.blocks()[0]
    assert int(b.src_ids[:b.n_dst].max()) < rows and int(b.nbr.max()) >= rows
    want = whole.clone()
    want[rows:] = whole[0]
    want = gmb.sage_forward_mx(blocks, want, mxw)
    csr.check_status()
    assert torch.equal(gmb.sage_forward_mx(blocks, whole[:rows], mxw), want)
    with pytest.raises(gmb.GmbError, match="ERANGE"):
        csr.check_status()
    gmb.sage_forward_mx(blocks, whole, mxw)
    csr.check_status()


# ---------------------------------------------------------------- training

def reference_step(host, x, ws, wn, bs, top, cls, labels, alpha, T):
    """Loss and gradients (weights, biases, input rows) of a distillation step
    in 64 bits: torch's differentiation on the CPU of the layers as Eq. (1)
    has them, from the loss's gradient by definition.  Also the smallest
    magnitude before a ReLU."""
    leaf = lambda a: torch.tensor(np.asarray(a, np.float64), requires_grad=True)  # noqa: E731
    x, ws, wn, bs = leaf(x), [leaf(a) for a in ws], [leaf(a) for a in wn], [leaf(a) for a in bs]
    h, least = x, np.inf
    for l, b in enumerate(host):
        ptr, idx = b.indptr.cpu().long(), b.indices.cpu().long()
        k = ptr[1:] - ptr[:-1]
        dst = torch.repeat_interleave(torch.arange(len(k)), k)
        m = torch.zeros(len(k), h.shape[1], dtype=torch.float64).index_add(0, dst, h[idx]) / k.clamp(min=1)[:, None]
        z = h[:len(k)] @ ws[l] + m @ wn[l] + bs[l]
        if l + 1 < len(host):
            least = min(least, float(z.detach().abs().min()))
            h = torch.relu(z)
    loss, grad, _ = mx_ref.distill(z.detach().numpy(), top, cls, labels, alpha, T)
    z.backward(torch.from_numpy(grad))
    return loss.mean(), [w.grad.numpy() for w in ws], [w.grad.numpy() for w in wn], [b.grad.numpy() for b in bs], \
        x.grad.numpy(), least


def teacher_of(rows, C, k, seed):
    rng = np.random.default_rng(seed)
    cls = np.stack([rng.permutation(C)[:k] for _ in range(rows)]).astype(np.int32)
    cls[rng.random(size=cls.shape) < 0.1] = -1
    top = (rng.normal(size=(rows, k)) * 2).astype(np.float32)
    labels = rng.integers(-1, C, size=rows).astype(np.int32)
    return top, cls, labels


def near(got, want, tol):
    err = np.abs(got.double().cpu().numpy() - want).max() / max(np.abs(want).max(), 1e-30)
    assert err <= tol, err


STEPS = [([20, 16, 8], [5, 5], 64, 0.5, 2.0, True), ([33, 24, 47], [6, 4], 100, 1.0, 1.0, False),
         ([16, 12, 12, 172], [4, 3, 3], 50, 0.7, 4.0, True), ([24, 601], [7], 90, 0.9, 2.0, True),
         ([24, 5000], [7], 30, 0.9, 2.0, True)]


# (embeddings: widths in whole fours, at most 640 columns above them)
@pytest.mark.parametrize("dims, fanouts, seeds, alpha, T, with_labels, embedding",
                         [(*s, False) for s in STEPS] + [(*STEPS[i], True) for i in (0, 2, 3)])
def test_backward_from_a_teacher(dg, graph, dims, fanouts, seeds, alpha, T, with_labels, embedding):
    """Weight gradients and the embedding rows' update against 64 bits: 2e-4 of
    each array's largest, the bound of this file's sums of up to a few thousand
    fp32 terms (no unit is near enough to its ReLU's corner to be decided
    otherwise, which is checked)."""
    g, csr = graph
    w = dg.sage_weights(dims, 3)
    wt = to_torch_weights(w)
    feats_np = dg.features(g.num_nodes, dims[0], 5, "f32")
    feats = torch.from_numpy(feats_np.copy()).cuda()
    ids = torch.from_numpy(dg.permutation(g.num_nodes, 9)[:seeds]).cuda()
    blocks = gmb.sample_blocks(csr, ids, fanouts, 4)
    x = gmb.gather_features(blocks, feats)
    fws = gmb._aligned_bytes(gmb.forward_workspace_bytes(blocks, wt), x.device)[1]
    logits = gmb.sage_forward(blocks, x, wt, workspace=fws)
    top, cls, labels = teacher_of(seeds, dims[-1], min(5, dims[-1]), 6)
    t = gmb.Teacher(torch.from_numpy(top).cuda(), torch.from_numpy(cls).cuda(), alpha, T)
    y = torch.from_numpy(labels).cuda() if with_labels else None
    lr = 10.0 * seeds
    grads, loss = gmb.sage_backward(blocks, x, wt, logits, y, fws, teacher=t,
                                    embedding=feats if embedding else None, emb_lr=lr)
    csr.check_status()
    host = blocks.blocks()
    src = host[0].src_ids.cpu().numpy()
    ws64, wn64, bs64 = w.as_f64()
    ref, dws, dwn, dbs, dx, least = reference_step(host, feats_np[src], ws64, wn64, bs64, top, cls,
                                                   labels if with_labels else None, alpha, T)
    assert least > 1e-6, least
    assert abs(float(loss) - ref) <= 1e-5 * max(1.0, abs(ref))
    for l in range(len(dims) - 1):
        near(grads.d_self[l], dws[l], 2e-4)
        near(grads.d_neigh[l], dwn[l], 2e-4)
        near(grads.d_bias[l], dbs[l], 2e-4)
    if embedding:
        want = feats_np.astype(np.float64)
        want[src] -= lr * dx
        moved = np.abs(want - feats_np).max()
        got = feats.double().cpu().numpy()
        assert np.abs(got - want).max() <= 2e-4 * moved + U32 * np.abs(want).max()
    # the loss operator by itself says the same of these logits
    alone, _ = gmb.distill_loss(logits, t.logits, t.classes, labels=y, alpha=alpha, temperature=T)
    assert abs(float(alone) - float(loss)) <= 4 * seeds * U32 * max(1.0, abs(float(loss)))


def test_a_bf16_student(dg, graph):
    """bf16 weights and features: the forward rounds means and hidden rows to
    bf16, as for the cross-entropy (2e-2)."""
    g, csr = graph
    dims = [32, 24, 40]
    w = dg.sage_weights(dims, 3)
    wt = gmb.SageWeights([torch.from_numpy(a).cuda().bfloat16() for a in w.w_self],
                         [torch.from_numpy(a).cuda().bfloat16() for a in w.w_neigh],
                         [torch.from_numpy(b).cuda() for b in w.bias])
    feats = torch.from_numpy(dg.features(g.num_nodes, 32, 5, "f32")).cuda().bfloat16()
    blocks = gmb.sample_blocks(csr, torch.arange(200, dtype=torch.int32, device="cuda"), [6, 5], 4)
    x = gmb.gather_features(blocks, feats)
    fws = gmb._aligned_bytes(gmb.forward_workspace_bytes(blocks, wt), x.device)[1]
    logits = gmb.sage_forward(blocks, x, wt, workspace=fws)
    top, cls, labels = teacher_of(200, 40, 6, 2)
    t = gmb.Teacher(torch.from_numpy(top).cuda(), torch.from_numpy(cls).cuda(), 0.6, 2.0)
    grads, loss = gmb.sage_backward(blocks, x, wt, logits, torch.from_numpy(labels).cuda(), fws, teacher=t)
    host = blocks.blocks()
    src = host[0].src_ids.cpu().numpy()
    f64 = lambda ts: [a.double().cpu().numpy() for a in ts]  # noqa: E731
    ref, dws, dwn, dbs, _, _ = reference_step(host, feats.double().cpu().numpy()[src], f64(wt.w_self), f64(wt.w_neigh),
                                              f64(wt.bias), top, cls, labels, 0.6, 2.0)
    assert abs(float(loss) - ref) <= 2e-2 * max(1.0, abs(ref))
    for l in range(2):
        near(grads.d_self[l], dws[l], 2e-2)
        near(grads.d_neigh[l], dwn[l], 2e-2)
        near(grads.d_bias[l], dbs[l], 2e-2)


def test_training_refusals_and_an_empty_batch(dg, graph):
    g, csr = graph
    dims = [16, 8]
    wt = to_torch_weights(dg.sage_weights(dims, 3))
    x = torch.randn(1000, 16, device="cuda")
    mk = lambda n, k=3: gmb.Teacher(torch.zeros(n, k, device="cuda"),  # noqa: E731
                                    torch.zeros(n, k, dtype=torch.int32, device="cuda"))
    empty = gmb.sample_blocks(csr, torch.empty(0, dtype=torch.int32, device="cuda"), [5], 3)
    fws = gmb._aligned_bytes(1 << 16, x.device)[1]
    logits = torch.empty(0, 8, device="cuda")
    grads, loss = gmb.sage_backward(empty, x, wt, logits, None, fws, teacher=mk(1))
    assert float(loss) == 0 and all(bool((a == 0).all()) for a in grads.d_self + grads.d_neigh + grads.d_bias)
    blocks = gmb.sample_blocks(csr, torch.arange(10, dtype=torch.int32, device="cuda"), [5], 3)
    logits = torch.zeros(10, 8, device="cuda")
    fws = gmb._aligned_bytes(gmb.forward_workspace_bytes(blocks, wt), x.device)[1]
    with pytest.raises(ValueError):
        gmb.sage_backward(blocks, x, wt, logits, None, fws, teacher=mk(9))
    with pytest.raises(TypeError):
        gmb.sage_backward(blocks, x, wt, logits, None, fws)
    with pytest.raises(TypeError):
        gmb.Teacher(torch.zeros(3, 3, device="cuda"), torch.zeros(3, 3, device="cuda"))


# ---------------------------------------------------------------- together

def test_a_student_in_four_bits(dg, graph):
    """A full-precision teacher's top logits train a model that is held in 4
    bits: its forward and backward run on what its records (and the store's)
    stand for, the step goes to fp32 masters, which are quantised again; then
    the records serve.  Also: vertices written back into the store."""
    g, csr = graph
    dims, fanouts, B = [64, 32, 20], [6, 5], 120
    feats_np = dg.features(g.num_nodes, dims[0], 5, "f32")
    feats = torch.from_numpy(feats_np).cuda()
    big = to_torch_weights(dg.sage_weights([64, 128, 20], 21))
    student = dg.sage_weights(dims, 3)
    masters = to_torch_weights(student)
    mxw = gmb.SageMxWeights(masters)
    table = gmb.mx_quantise(feats, gmb.MXFP4)
    for step in range(2):
        ids = torch.from_numpy(dg.permutation(g.num_nodes, 30 + step)[:B]).cuda()
        blocks = gmb.sample_blocks(csr, ids, fanouts, step)
        taught = gmb.sage_forward_fused(blocks, feats, big)[0]
        top, cls = torch.topk(taught, 4)
        t = gmb.Teacher(top.contiguous(), cls.int().contiguous(), 1.0, 2.0)
        w = mxw.values()
        x = gmb.mx_gather(blocks, table, dims[0], gmb.MXFP4)
        fws = gmb._aligned_bytes(gmb.forward_workspace_bytes(blocks, w), x.device)[1]
        logits = gmb.sage_forward(blocks, x, w, workspace=fws)
        grads, loss = gmb.sage_backward(blocks, x, w, logits, None, fws, teacher=t)
        host = blocks.blocks()
        src = host[0].src_ids.cpu().numpy()
        stored = mx_ref.values(table.cpu().numpy()[src], dims[0], 4)
        f64 = lambda ts: [a.double().cpu().numpy() for a in ts]  # noqa: E731
        for l in range(2):   # what the student computes with is what its records say
            rec = mxw.w_self[l].cpu().numpy()
            assert np.array_equal(w.w_self[l].cpu().numpy(), mx_ref.values(rec, dims[l], 4).T.astype(np.float32))
        ref, dws, dwn, dbs, _, least = reference_step(host, stored, f64(w.w_self), f64(w.w_neigh), f64(w.bias),
                                                      top.cpu().numpy(), cls.int().cpu().numpy(), None, 1.0, 2.0)
        assert least > 1e-7, least
        assert abs(float(loss) - ref) <= 1e-5 * max(1.0, abs(ref))
        for l in range(2):
            near(grads.d_self[l], dws[l], 2e-4)
            near(grads.d_neigh[l], dwn[l], 2e-4)
            near(grads.d_bias[l], dbs[l], 2e-4)
        before = [a.clone() for a in masters.w_self]
        gmb.sgd_update(masters, grads, 0.5)
        assert all(not torch.equal(a, b) for a, b in zip(before, masters.w_self))
        mxw.requantise(masters)
        for l in range(2):
            assert np.array_equal(mxw.w_neigh[l].cpu().numpy(), mx_ref.quantise(masters.w_neigh[l].t().cpu().numpy(), 4))
        served(blocks, table, masters, mxw)
        # the batch's rows, changed, go back into the store
        rows = x.clone()
        rows *= 1.25
        gmb.mx_quantise(rows, gmb.MXFP4, ids=blocks, table=table)
        changed = mx_ref.quantise(rows[:len(src)].cpu().numpy(), 4)
        assert np.array_equal(table.cpu().numpy()[src], changed)
    csr.check_status()


def test_a_captured_step_and_two_graphs_of_one_workspace(dg, graph):
    """A training step from the records to the records again as one graph, and
    the serving of two batches as two graphs of one workspace, replayed in
    turn: each replay gives what the eager calls give (the step's sums in
    another order)."""
    g, csr = graph
    dims, fanouts, B = [64, 32, 20], [6, 5], 90
    masters = to_torch_weights(dg.sage_weights(dims, 3))
    mxw = gmb.SageMxWeights(masters)
    feats = torch.from_numpy(dg.features(g.num_nodes, dims[0], 5, "f32")).cuda()
    table = gmb.mx_quantise(feats, gmb.MXFP4)
    batches = [gmb.sample_blocks(csr, torch.from_numpy(dg.permutation(g.num_nodes, s)[:B]).cuda(), fanouts, s)
               for s in (1, 2)]
    top, cls, labels = teacher_of(B, 20, 4, 8)
    top, y = torch.from_numpy(top).cuda(), torch.from_numpy(labels).cuda()
    t = gmb.Teacher(top, torch.from_numpy(cls).cuda(), 0.5, 2.0)
    x = gmb.mx_gather(batches[0], table, dims[0], gmb.MXFP4)
    w = mxw.values()
    aligned = lambda n: gmb._aligned_bytes(n, x.device)[1]  # noqa: E731
    fws, bws = aligned(gmb.forward_workspace_bytes(batches[0], w)), aligned(gmb.backward_workspace_bytes(batches[0], w))
    logits, loss, grads = torch.empty(B, 20, device="cuda"), torch.empty(1, device="cuda"), gmb.SageGrads(w)

    def step():
        gmb.mx_gather(batches[0], table, dims[0], gmb.MXFP4, out=x)
        for l in range(2):
            w.w_self[l].copy_(gmb.mx_gather(None, mxw.w_self[l], dims[l], gmb.MXFP4).t())
            w.w_neigh[l].copy_(gmb.mx_gather(None, mxw.w_neigh[l], dims[l], gmb.MXFP4).t())
        gmb.sage_forward(batches[0], x, w, logits=logits, workspace=fws)
        gmb.sage_backward(batches[0], x, w, logits, y, fws, grads=grads, loss=loss, workspace=bws, teacher=t)
        gmb.sgd_update(masters, grads, 0.5)
        mxw.requantise(masters)

    step()                                       # (first uses, outside the graph)
    torch.cuda.synchronize()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg):
        step()
    params = [a for ms in (masters.w_self, masters.w_neigh, masters.bias) for a in ms]
    for seed in range(3):
        top.copy_(torch.from_numpy(teacher_of(B, 20, 4, seed)[0]))
        start = [a.clone() for a in params]
        mxw.requantise(masters)
        step()
        want, exact = [a.clone() for a in params], [loss.clone(), logits.clone()]
        for a, b in zip(params, start):
            a.copy_(b)
        mxw.requantise(masters)
        torch.cuda.synchronize()
        cg.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([loss, logits], exact))
        # (the mean's backward adds a row's edges in the order in which they
        # arrived: each side is within this file's 2e-4 of the exact step, and
        # rounds the new value once)
        for a, b, c in zip(params, want, start):
            assert float((a - b).abs().max()) <= 4e-4 * float((b - c).abs().max()) + 2 * U32 * float(b.abs().max())
        for l in range(2):
            assert np.array_equal(mxw.w_self[l].cpu().numpy(), mx_ref.quantise(masters.w_self[l].t().cpu().numpy(), 4))
        assert any(not torch.equal(a, b) for a, b in zip(params, start))
    ws = aligned(max(gmb.mx_forward_workspace_bytes(b, mxw) for b in batches))
    outs = [torch.empty(B, 20, device="cuda") for _ in batches]
    graphs = []
    for b, o in zip(batches, outs):
        gmb.sage_forward_mx(b, table, mxw, workspace=ws, logits=o)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            gmb.sage_forward_mx(b, table, mxw, workspace=ws, logits=o)
    want = [gmb.sage_forward_mx(b, table, mxw) for b in batches]
    for _ in range(3):
        for o in outs:
            o.zero_()
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, v) for o, v in zip(outs, want))
    csr.check_status()
