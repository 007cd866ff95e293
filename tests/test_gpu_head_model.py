"""Dropout inside the model, and a whole training step as the operators are used
together, against 64 bits: blocks, forward with dropout, norm with a residual,
cross-entropy over many classes, and back down to the weights and embeddings.

Bounds: the model's forward and gradients are within 1e-5 of the largest value
here (fp32; products of widths up to 64 and means of up to 10 rows, each a few
half-steps of 2^-24 of its terms, through three layers)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU on this machine", allow_module_level=True)

import head_ref  # noqa: E402
import paper_2010_05337_amd as gmb  # noqa: E402
from datagen.configs import make_workload  # noqa: E402

EPS = 1e-5


@pytest.fixture(scope="module")
def tiny():
    wl = make_workload("tiny")
    g = wl.graph
    csr = gmb.CSRGraph(torch.from_numpy(g.indptr.astype(np.int32)).cuda(), torch.from_numpy(g.indices).cuda())
    return wl, csr


def weights(dims, seed, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    mat = lambda a, b: (torch.randn(a, b, generator=gen) / a ** 0.5).to(dtype).cuda()  # noqa: E731
    pairs = list(zip(dims, dims[1:]))
    return gmb.SageWeights([mat(a, b) for a, b in pairs], [mat(a, b) for a, b in pairs],
                           [(torch.randn(b, generator=gen) * 0.1).cuda() for _, b in pairs])


class Reference:
    """The model in 64 bits with torch's own gradients."""

    def __init__(self, blocks, w, drop):
        self.blocks = blocks.blocks()
        self.par = [[t.double().cpu().requires_grad_() for t in ts] for ts in (w.w_self, w.w_neigh, w.bias)]
        self.drop = drop

    def forward(self, x):
        h, L = x, len(self.blocks)
        for l, b in enumerate(self.blocks):
            ptr, idx = b.indptr.long().cpu(), b.indices.long().cpu()
            k = ptr[1:] - ptr[:-1]
            dst = torch.repeat_interleave(torch.arange(b.n_dst), k)
            mean = torch.zeros(b.n_dst, h.shape[1], dtype=torch.float64).index_add(0, dst, h[idx]) / k.clamp(min=1)[:, None]
            h = h[:b.n_dst] @ self.par[0][l] + mean @ self.par[1][l] + self.par[2][l]
            if l < L - 1:
                h = torch.relu(h)
                if self.drop is not None:
                    d = self.drop
                    kept = head_ref.keep(b.src_ids[:b.n_dst].cpu().numpy(), h.shape[1], d.p, d.seed, d.layer + l)
                    h = head_ref.drop(h, kept, d.p)
        return h


def near(got, want, what, tol=1e-5):
    got, want = got.double().cpu(), want.detach()
    err = (got - want).abs().max().item() / max(want.abs().max().item(), 1e-30)
    assert err <= tol, (what, err)


def sample(tiny, n=64, seed=5, fanouts=(5, 5)):
    wl, csr = tiny
    seeds = torch.from_numpy(wl.batches[0][:n].copy()).cuda()
    return csr, seeds, gmb.sample_blocks(csr, seeds, list(fanouts), seed)


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.5, 0.9, 1.0])
@pytest.mark.parametrize("dims, fanouts", [((16, 32, 8), (5, 5)), ((16, 64, 32, 20), (4, 3, 5)), ((16, 8), (5,))], ids=str)
def test_model_with_dropout(tiny, dims, fanouts, p, fused):
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny, fanouts=fanouts)
    w = weights(dims, 1)
    feats = torch.from_numpy(wl.feats).cuda()
    d = gmb.Dropout(p, 1234567890123, layer=3)
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    if fused:
        out, x = gmb.sage_forward_fused(blocks, feats, w, workspace=ws, dropout=d)
    else:
        x = gmb.gather_features(blocks, feats)
        out = gmb.sage_forward(blocks, x, w, workspace=ws, dropout=d)
    ref = Reference(blocks, w, d)
    n_src = blocks.sizes()[0][1]
    rows = feats[blocks.input_ids[:n_src].long()].double().cpu().requires_grad_()
    want = ref.forward(rows)
    near(out, want, "outputs")
    dy = torch.randn(out.shape, generator=torch.Generator().manual_seed(2))
    want.backward(dy.double())
    grads = gmb.sage_backward_from(blocks, x, w, dy.cuda(), ws, dropout=d)
    for l in range(len(dims) - 1):
        for got, par, name in ((grads.d_self, 0, "self"), (grads.d_neigh, 1, "neigh"), (grads.d_bias, 2, "bias")):
            g = ref.par[par][l].grad
            near(got[l], g if g is not None else torch.zeros(got[l].shape, dtype=torch.float64), (name, l))
    # the embeddings' step
    table = feats.clone()
    again = gmb.sage_backward_from(blocks, x, w, dy.cuda(), ws, dropout=d, embedding=table, emb_lr=0.5)
    step = (feats - table)[blocks.input_ids[:n_src].long()]
    near(step, 0.5 * rows.grad, "embeddings", tol=1e-4)       # (a difference of fp32 rows: a half-step of theirs)
    near(again.d_self[-1], ref.par[0][-1].grad, "again")
    csr.check_status()


def test_without_dropout_it_is_the_old_path(tiny):
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny)
    w = weights((16, 32, 8), 3)
    x = gmb.gather_features(blocks, torch.from_numpy(wl.feats).cuda())
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    out = gmb.sage_forward(blocks, x, w, workspace=ws)
    assert torch.equal(gmb.sage_forward(blocks, x, w, dropout=gmb.Dropout(0.0, 7)), out)
    labels = torch.arange(64, dtype=torch.int32, device="cuda") % 8
    grads, _ = gmb.sage_backward(blocks, x, w, out, labels, ws)
    _, g = gmb.distill_loss(out, torch.zeros(64, 1, device="cuda"), torch.full((64, 1), -1, dtype=torch.int32, device="cuda"),
                            labels=labels, alpha=0.0)
    mine = gmb.sage_backward_from(blocks, x, w, g, ws)
    for l in range(2):
        near(mine.d_self[l], grads.d_self[l].double().cpu(), l)
        near(mine.d_neigh[l], grads.d_neigh[l].double().cpu(), l)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_a_bf16_model_with_dropout(tiny, dtype):
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny)
    w = weights((16, 32, 8), 4, dtype)
    x = gmb.gather_features(blocks, torch.from_numpy(wl.feats).cuda().to(dtype))
    d = gmb.Dropout(0.5, 99)
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    out, hidden = gmb.sage_forward(blocks, x, w, workspace=ws, dropout=d, return_hidden=True)
    plain, before = gmb.sage_forward(blocks, x, w, return_hidden=True)
    n_dst = blocks.sizes()[0][0]
    ids = blocks.input_ids[:n_dst].contiguous()
    assert torch.equal(hidden[0], gmb.dropout(before[0].contiguous(), d, ids=ids))
    grads = gmb.sage_backward_from(blocks, x, w, torch.ones_like(out), ws, dropout=d)
    assert all(bool(t.isfinite().all()) for t in grads.d_self + grads.d_neigh + grads.d_bias)


def test_dropout_is_a_dropout(tiny):
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny)
    w = weights((16, 32, 8), 3)
    feats = torch.from_numpy(wl.feats).cuda()
    x = gmb.gather_features(blocks, feats)
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    out = gmb.sage_forward(blocks, x, w, workspace=ws)
    for call in [lambda: gmb.sage_forward(blocks, x, w, dropout=0.5), lambda: gmb.sage_forward_fused(blocks, feats, w, dropout=0.5),
                 lambda: gmb.sage_backward_from(blocks, x, w, out, ws, dropout=0.5)]:
        with pytest.raises(TypeError):
            call()


def head_step(blocks, x, w, ws, drop, gain, table, labels, model_drop):
    """One pass of a residual head on the model: outputs h, r = h + dropout(h turned), its norm, the loss over the table's rows."""
    h = gmb.sage_forward(blocks, x, w, workspace=ws, dropout=model_drop)
    y, r = gmb.rms_norm(h, gain, EPS, residual=h, dropout=drop)
    loss, g = gmb.linear_loss(y, table, labels)
    n = gmb.rms_norm_backward(g.x, r, gain, EPS, dropout=drop)
    dh = n.x + n.residual
    return loss, gmb.sage_backward_from(blocks, x, w, dh, ws, dropout=model_drop), n.weight, g.w, y


def test_a_training_step_through_all_of_them(tiny):
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny)
    w = weights((16, 32, 24), 5)
    feats = torch.from_numpy(wl.feats).cuda()
    x = gmb.gather_features(blocks, feats)
    gen = torch.Generator().manual_seed(6)
    table = torch.randn(700, 24, generator=gen).cuda()          # 700 vertices, each a class
    gain = (1 + 0.1 * torch.randn(24, generator=gen)).cuda()
    labels = torch.randint(-1, 700, (64,), generator=gen).int().cuda()
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    drop, model_drop = gmb.Dropout(0.25, 17, layer=9), gmb.Dropout(0.5, 17)
    loss, grads, d_gain, d_table, y = head_step(blocks, x, w, ws, drop, gain, table, labels, model_drop)

    ref = Reference(blocks, w, model_drop)
    n_src = blocks.sizes()[0][1]
    h = ref.forward(feats[blocks.input_ids[:n_src].long()].double().cpu())
    G, T = gain.double().cpu().requires_grad_(), table.double().cpu().requires_grad_()
    r = h + head_ref.drop(h, head_ref.keep(np.arange(64), 24, 0.25, 17, 9), 0.25)
    z = head_ref.rms_norm(r, G, EPS) @ T.t()
    on = labels.cpu() >= 0
    want = torch.nn.functional.cross_entropy(z[on], labels.cpu()[on].long(), reduction="sum") / 64
    want.backward()
    near(loss, want.reshape(1), "loss")
    near(d_gain, G.grad, "gain")
    near(d_table, T.grad, "table")
    for l in range(2):
        near(grads.d_self[l], ref.par[0][l].grad, ("self", l), tol=2e-5)
        near(grads.d_neigh[l], ref.par[1][l].grad, ("neigh", l), tol=2e-5)
        near(grads.d_bias[l], ref.par[2][l].grad, ("bias", l), tol=2e-5)
    # served: the norm's rows in the 8-bit store
    rec, _ = gmb.rms_norm(gmb.sage_forward(blocks, x, w), gain, EPS, bits=8)
    assert rec.shape == (64, gmb.mx_row_bytes(24, 8))
    csr.check_status()


def test_a_captured_training_step(tiny):
    """The same step as a graph, its dropout's step on the device, while eager calls run between the replays."""
    wl, _ = tiny
    csr, seeds, blocks = sample(tiny)
    w = weights((16, 32, 24), 7)
    x = gmb.gather_features(blocks, torch.from_numpy(wl.feats).cuda())
    gen = torch.Generator().manual_seed(8)
    table, gain = torch.randn(300, 24, generator=gen).cuda(), torch.ones(24, device="cuda")
    labels = torch.randint(-1, 300, (64,), generator=gen).int().cuda()
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    counter = torch.zeros(1, dtype=torch.int32, device="cuda")
    drop, model_drop = gmb.Dropout(0.25, 1, layer=9, step=counter), gmb.Dropout(0.5, 1, step=counter)
    args = (blocks, x, w, ws, drop, gain, table, labels, model_drop)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        head_step(*args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = head_step(*args)
    losses = set()
    for k in (0, 1, 2, 2):
        counter.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        have = [got[0].clone(), got[2].clone(), got[3].clone(), got[1].d_self[-1].clone()]
        want = head_step(*args)
        for a, b in zip(have, (want[0], want[2], want[3], want[1].d_self[-1])):
            assert torch.equal(a, b), k
        losses.add(have[0].item())
    assert len(losses) == 3


def test_an_empty_batch(tiny):
    wl, csr = tiny
    blocks = gmb.sample_blocks(csr, torch.empty(0, dtype=torch.int32, device="cuda"), [5, 5], 1)
    w = weights((16, 32, 8), 9)
    x = torch.zeros(max(blocks.input_capacity, 1), 16, device="cuda")
    ws = torch.empty(gmb.forward_workspace_bytes(blocks, w), dtype=torch.uint8, device="cuda")
    out = gmb.sage_forward(blocks, x, w, workspace=ws, dropout=gmb.Dropout(0.5, 1))
    assert out.shape == (0, 8)
    grads = gmb.sage_backward_from(blocks, x, w, out, ws, dropout=gmb.Dropout(0.5, 1))
    assert not any(t.any() for t in grads.d_self + grads.d_neigh + grads.d_bias)
