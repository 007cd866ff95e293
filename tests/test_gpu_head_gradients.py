"""The model's gradients under dropout from the hidden rows that its forward
left, for fp32 and bf16 models, and which backward a forward with dropout takes.

Bounds.  Given the stored hidden rows the backward is a chain of linear maps in
fp32: sums of at most 64 columns, 10 edges and 64 destinations, three layers of
them, 1e-5 of the largest value of a result (as in test_gpu_head_model.py).  In
a bf16 model the neighbours' mean is stored in bf16: half a step, 2^-8, of every
term of its product."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import head_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402
from test_gpu_head_model import sample, tiny, weights  # noqa: E402, F401

TYPES = [torch.float32, torch.bfloat16]


def reference(blocks, w, x, hidden, dz, p):
    """[(dW_self, dW_neigh, db, |mean|^T |dZ|)] a layer, in 64 bits, from x, the dropped hidden rows and dZ of the last layer."""
    out = []
    scale = 65536 / (65536 - int(65536 * p + 0.5))
    for l in reversed(range(len(hidden) + 1)):
        b = blocks[l]
        h = (x if l == 0 else hidden[l - 1]).double().cpu()[:b.n_src]
        ptr, idx = b.indptr.long().cpu(), b.indices.long().cpu()
        k = ptr[1:] - ptr[:-1]
        dst = torch.repeat_interleave(torch.arange(b.n_dst), k)
        per = 1 / k.clamp(min=1).double()
        mean = torch.zeros(b.n_dst, h.shape[1], dtype=torch.float64).index_add(0, dst, h[idx]) * per[:, None]
        out.insert(0, (h[:b.n_dst].t() @ dz, mean.t() @ dz, dz.sum(0), mean.abs().t() @ dz.abs()))
        if l:
            d = torch.zeros_like(h)
            d[:b.n_dst] += dz @ w.w_self[l].double().cpu().t()
            d.index_add_(0, idx, (dz * per[:, None] @ w.w_neigh[l].double().cpu().t())[dst])
            dz = d * scale * (h > 0)
    return out


def near(got, want, more, what):
    got = got.double().cpu()
    err = (got - want).abs() - more
    assert float(err.max()) <= 1e-5 * float(want.abs().max()), (what, float(err.max()), float(want.abs().max()))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("p", [0.0, 0.5, 0.9])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dims, fanouts", [((16, 64, 32, 20), (4, 3, 5)), ((16, 32, 8), (5, 5))], ids=str)
def test_gradients_from_the_stored_rows(tiny, dims, fanouts, fused, p, dtype):  # noqa: F811
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny, fanouts=fanouts)
    w = weights(dims, 11, dtype)
    feats = torch.from_numpy(wl.feats).cuda().to(dtype)
    x = gmb.gather_features(blocks, feats)
    d = gmb.Dropout(p, 77, layer=2)
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    if fused:
        out, x_dst, hidden = gmb.sage_forward_fused(blocks, feats, w, workspace=ws, return_hidden=True, dropout=d)
    else:
        out, hidden = gmb.sage_forward(blocks, x, w, workspace=ws, return_hidden=True, dropout=d)
    made = blocks.blocks()
    for l, h in enumerate(hidden):                   # the mask: what the generator drops is 0
        kept = head_ref.keep(made[l].src_ids[:made[l].n_dst].cpu().numpy(), h.shape[1], p, 77, 2 + l)
        assert not h.cpu()[~kept].any() and bool((h.cpu()[kept] > 0).any())
    dy = torch.randn(out.shape, generator=torch.Generator().manual_seed(12))
    grads = gmb.sage_backward_from(blocks, x_dst if fused else x, w, dy.cuda(), ws, dropout=d)
    for l, (ws_, wn, b, size) in enumerate(reference(made, w, x, hidden, dy.double(), p)):
        near(grads.d_self[l], ws_, 0, ("self", l))
        near(grads.d_neigh[l], wn, 2.0 ** -8 * size if dtype is torch.bfloat16 else 0, ("neigh", l))
        near(grads.d_bias[l], b, 0, ("bias", l))
    csr.check_status()


def test_a_backward_takes_the_forwards_dropout(tiny):  # noqa: F811
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny)
    w = weights((16, 32, 8), 13)
    feats = torch.from_numpy(wl.feats).cuda()
    x = gmb.gather_features(blocks, feats)
    labels = torch.zeros(64, dtype=torch.int32, device="cuda")
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    d = gmb.Dropout(0.5, 3)
    teacher = gmb.Teacher(torch.zeros(64, 1, device="cuda"), torch.zeros(64, 1, dtype=torch.int32, device="cuda"))
    for forward in (lambda **k: gmb.sage_forward(blocks, x, w, workspace=ws, **k),
                    lambda **k: gmb.sage_forward_fused(blocks, feats, w, workspace=ws, **k)[0]):
        out = forward(dropout=d)
        for call in (lambda: gmb.sage_backward(blocks, x, w, out, labels, ws),
                     lambda: gmb.sage_backward(blocks, x, w, out, labels, ws, embedding=feats.clone(), emb_lr=0.1),
                     lambda: gmb.sage_backward(blocks, x, w, out, labels, ws, teacher=teacher),
                     lambda: gmb.sage_backward_from(blocks, x, w, out, ws),
                     lambda: gmb.sage_backward_from(blocks, x, w, out, ws, dropout=gmb.Dropout(0.25, 3))):
            with pytest.raises(ValueError):
                call()
        gmb.sage_backward_from(blocks, x, w, out, ws, dropout=d)
        # nothing was dropped: any of them
        out = forward(dropout=gmb.Dropout(1e-6, 3))
        gmb.sage_backward(blocks, x, w, out, labels, ws)
        out = forward()
        gmb.sage_backward(blocks, x, w, out, labels, ws)
        gmb.sage_backward_from(blocks, x, w, out, ws)
        with pytest.raises(ValueError):
            gmb.sage_backward_from(blocks, x, w, out, ws, dropout=d)
    # a model without hidden rows has nothing to drop
    csr, seeds, blocks = sample(tiny, fanouts=(5,))
    w = weights((16, 8), 14)
    x = gmb.gather_features(blocks, feats)
    ws = torch.empty(max(gmb.forward_workspace_bytes(blocks, w), 256), dtype=torch.uint8, device="cuda")
    out = gmb.sage_forward(blocks, x, w, workspace=ws, dropout=d)
    a, _ = gmb.sage_backward(blocks, x, w, out, labels, ws)
    assert bool(a.d_self[0].isfinite().all())
    csr.check_status()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(5, 7), (64, 16), (257, 100), (9, 257), (3, 8200)], ids=str)
def test_the_backward_of_dropout_is_its_adjoint(shape, dtype):
    """<dropout(x), dy> = <x, dropout(dy)>, element by element: the mask and factor of the definition on either side."""
    n, dim = shape
    gen = torch.Generator().manual_seed(15)
    x, dy = (torch.randn(n, dim, generator=gen).to(dtype) for _ in range(2))
    ids = torch.randint(0, 1 << 31, (n,), dtype=torch.int64, generator=gen).int()
    for p, seed, layer in [(0.5, 1, 0), (0.1, 2, 5)]:
        d = gmb.Dropout(p, seed, layer)
        y = gmb.dropout(x.cuda(), d, ids=ids.cuda()).double().cpu()
        dx = gmb.dropout(dy.cuda(), d, ids=ids.cuda()).double().cpu()
        kept = head_ref.keep(ids.numpy(), dim, p, seed, layer)
        want = head_ref.drop(dy.double(), kept, p)
        # the factor's and the product's rounding, and the result's in bf16
        tol = (2 * 2.0 ** -24 + (2.0 ** -8 if dtype is torch.bfloat16 else 0)) * 1.001 * want.abs()
        assert bool(((dx - want).abs() <= tol).all())
        a, b = y * dy.double(), x.double() * dx
        assert bool(((a - b).abs() <= 2 * tol.max() / want.abs().max() * a.abs().maximum(b.abs())).all())
