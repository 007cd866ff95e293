"""Refusals of the dropout's, norm's and linear loss's entry points and of the
model's with dropout: bad arguments are found on the host, before anything is
enqueued (addresses here are never read)."""
import ctypes
import os

import pytest

EINVAL, ENOSPC = -1, -2
P = 1 << 40          # an aligned address that nothing reads
Q = P + (1 << 36)    # and others, far apart
R = Q + (1 << 36)
S = R + (1 << 36)


@pytest.fixture(scope="module")
def gmb():
    import paper_2010_05337_amd as gmb
    if not os.path.exists(gmb.LIB_PATH):
        from paper_2010_05337_amd import build
        build.build()
    gmb.lib()
    return gmb


def rows(gmb, at, stride):
    return None if at is False else gmb.RowsStruct(at, stride)


def drop(gmb, p=0.5, layer=0, none=False):
    return None if none else gmb.DropoutStruct(1, p, layer, None)


def dropout(gmb, x=P, xs=100, res=False, rs=100, out=Q, os_=100, n=10, dim=100, dtype=0, **d):
    return gmb.lib().gmb_dropout_rows(rows(gmb, x, xs), rows(gmb, res, rs), drop(gmb, **d), None, None, n, dim, dtype,
                                      rows(gmb, out, os_), None)


SHAPE = [dict(n=-1), dict(n=1 << 31), dict(dim=0), dict(dim=65537, xs=1 << 17), dict(dtype=2), dict(dtype=-1)]


@pytest.mark.parametrize("bad", SHAPE + [
    dict(x=None), dict(x=False), dict(xs=99), dict(out=None), dict(out=False), dict(os_=99), dict(res=None), dict(res=R, rs=99),
    dict(out=P, os_=104), dict(res=R, out=R, os_=104), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(layer=-1),
    dict(none=True)], ids=str)
def test_dropout_refuses(gmb, bad):
    assert dropout(gmb, **bad) == EINVAL
    assert gmb.lib().gmb_last_error()


def test_no_rows_need_no_pointers(gmb):
    assert dropout(gmb, n=0, x=False, out=False) == 0
    assert norm(gmb, n=0, x=False, out=False) == 0


def norm(gmb, x=P, xs=100, res=False, rs=100, total=False, ts=100, out=Q, os_=100, n=10, dim=100, dtype=0, weight=None,
         eps=1e-6, fmt=0, none=True, **d):
    return gmb.lib().gmb_rms_norm(rows(gmb, x, xs), rows(gmb, res, rs), drop(gmb, none=none, **d), None, None, n, dim, dtype,
                                  weight, eps, rows(gmb, total, ts), fmt, rows(gmb, out, os_), None)


@pytest.mark.parametrize("bad", SHAPE + [
    dict(x=None), dict(x=False), dict(xs=99), dict(out=None), dict(out=False), dict(os_=99), dict(res=None), dict(res=R, rs=99),
    dict(total=R, ts=99), dict(total=P, ts=101), dict(res=R, total=R, ts=101), dict(total=Q), dict(out=P, os_=101),
    dict(eps=0.0), dict(eps=1e-38), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(fmt=5), dict(fmt=-4),
    dict(fmt=8, os_=128), dict(fmt=8, os_=143), dict(fmt=8, os_=144, out=Q + 8), dict(fmt=4, os_=64), dict(fmt=8, os_=144, out=P),
    dict(fmt=8, os_=144, res=R, out=R), dict(none=False, p=2.0), dict(none=False, layer=-3)], ids=str)
def test_norm_refuses(gmb, bad):
    assert norm(gmb, **bad) == EINVAL
    assert gmb.lib().gmb_last_error()


def test_norm_workspace(gmb):
    L = gmb.lib()
    assert L.gmb_rms_norm_workspace_bytes(-1, 4) == 0 and L.gmb_rms_norm_workspace_bytes(4, 0) == 0
    assert L.gmb_rms_norm_workspace_bytes(4, 65537) == 0 and L.gmb_rms_norm_workspace_bytes(1 << 31, 4) == 0
    assert L.gmb_rms_norm_workspace_bytes(0, 4) >= 16


def back(gmb, dy=P, dys=100, r=Q, rs=100, carry=False, cs=100, d_res=R, ds=100, dx=False, xs=100, n=10, dim=100, dtype=0,
         weight=None, eps=1e-6, dw=None, ws=None, ws_bytes=0, none=True, **d):
    return gmb.lib().gmb_rms_norm_backward(rows(gmb, dy, dys), rows(gmb, r, rs), rows(gmb, carry, cs), drop(gmb, none=none, **d),
                                           None, None, n, dim, dtype, weight, eps, rows(gmb, d_res, ds), rows(gmb, dx, xs), dw,
                                           ws, ws_bytes, None)


@pytest.mark.parametrize("bad", SHAPE + [
    dict(dy=None), dict(dy=False), dict(dys=99), dict(r=None), dict(r=False), dict(rs=99), dict(carry=None), dict(carry=S, cs=99),
    dict(d_res=None), dict(ds=99), dict(dx=None), dict(dx=S, xs=99), dict(d_res=P, ds=101), dict(d_res=Q, ds=101),
    dict(dx=Q, xs=101), dict(dx=R), dict(carry=S, dx=S, xs=101), dict(eps=0.0), dict(eps=1e-38), dict(none=False, p=-1.0),
    dict(dw=S), dict(dw=S, ws=P + 16, ws_bytes=1 << 30)], ids=str)
def test_norm_backward_refuses(gmb, bad):
    assert back(gmb, **bad) == EINVAL
    assert gmb.lib().gmb_last_error()


def test_norm_backward_refuses_a_small_workspace(gmb):
    need = gmb.lib().gmb_rms_norm_workspace_bytes(10, 100)
    assert back(gmb, dw=S, ws=P, ws_bytes=need - 1) == ENOSPC


def loss(gmb, x=P, xs=64, w=Q, wr=64, wc=1, bias=None, labels=R, n=10, d=64, classes=100, dtype=0, dx=None, dw=None, db=None,
         turned=0, out=S, ws=None, ws_bytes=0, size_only=False, none=False):
    head = None if none else gmb.LinearHeadStruct(x, xs, w, wr, wc, bias, labels, n, d, classes, dtype, 0)
    grads = gmb.LinearGradsStruct(dx, dw, db, turned, 0)
    if size_only:
        return gmb.lib().gmb_linear_loss_workspace_bytes(head, grads)
    return gmb.lib().gmb_linear_loss(head, grads, out, ws, ws_bytes, None)


HEAD = [dict(none=True), dict(n=-1), dict(n=(1 << 22) + 1), dict(d=0), dict(d=65537, xs=1 << 17), dict(classes=0),
        dict(classes=(1 << 27) + 1), dict(dtype=2), dict(xs=63), dict(wr=-1), dict(wc=-1)]


@pytest.mark.parametrize("bad", HEAD + [
    dict(x=None), dict(w=None), dict(labels=None), dict(out=None), dict(ws=None), dict(ws=P + 16, ws_bytes=1 << 30),
    dict(dx=P), dict(dx=P + 2000), dict(dw=Q), dict(dw=Q - 100), dict(bias=S + 4096, db=S + 4096), dict(dx=R), dict(db=Q + 64)], ids=str)
def test_linear_loss_refuses(gmb, bad):
    assert loss(gmb, **bad) == EINVAL
    assert gmb.lib().gmb_last_error()


@pytest.mark.parametrize("bad", HEAD, ids=str)
def test_linear_loss_bytes_refuses(gmb, bad):
    assert loss(gmb, size_only=True, **bad) == 0


def test_linear_loss_refuses_a_small_workspace(gmb):
    need = loss(gmb, size_only=True)
    assert need > 0 and loss(gmb, ws=P, ws_bytes=need - 1) == ENOSPC
    grads = dict(dx=S + (1 << 30), dw=S + (1 << 31), db=S + (3 << 30))
    assert loss(gmb, size_only=True, **grads) >= need    # (one launch, nothing in between)
    assert loss(gmb, size_only=True, n=2000, classes=5000, **grads) > loss(gmb, size_only=True, n=2000, classes=5000)


@pytest.mark.parametrize("big", [
    dict(n=1 << 22, d=65536, xs=65536, wr=65536, classes=1000, dx=S, dw=S), dict(n=100, d=65536, xs=65536, wr=65536, classes=1 << 27),
    dict(n=1 << 22, d=65536, xs=65536, wr=65536, classes=1 << 27, dtype=1, dx=S, dw=S)], ids=str)
def test_linear_loss_refuses_what_no_launch_takes(gmb, big):
    # more 64 x 64 tiles than a launch has workgroups: said before anything is launched
    assert loss(gmb, size_only=True, **big) == 0
    apart = {k: v if k not in ("dx", "dw") else 1 << 60 for k, v in big.items()}
    assert loss(gmb, ws=P, ws_bytes=1 << 60, **apart) == EINVAL
    assert b"too many together" in gmb.lib().gmb_last_error()


def test_linear_loss_workspace_is_bounded(gmb):
    # a hundred million classes for a thousand rows: no room for the logits (200 GB), 384 MB of gradients at a time
    need = loss(gmb, size_only=True, n=1000, d=128, xs=128, wr=128, classes=100_000_000, dtype=1, dx=S, dw=S)
    assert need < 8 << 30


@pytest.fixture()
def model(gmb):
    b, w, g = gmb.BlocksStruct(), gmb.WeightsStruct(), gmb.GradsStruct()
    b.num_layers = w.num_layers = g.num_layers = 2
    b.num_seeds = 4
    for l, (dst, src) in enumerate([(8, 32), (4, 8)]):
        k = b.blk[l]
        k.indptr = k.indices = k.nbr = k.src_ids = k.sizes = P
        k.cap_dst, k.cap_src, k.cap_nnz, k.fanout, k.layer = dst, src, src, 4, l
        w.w_self[l] = w.w_neigh[l] = w.bias[l] = P
        g.d_self[l] = g.d_neigh[l] = g.d_bias[l] = P
    w.dims[0], w.dims[1], w.dims[2] = 16, 16, 8
    return b, w, g


def forward(gmb, m, x=P, feats=None, nodes=0, logits=P, ws=P, ws_bytes=1 << 40, **d):
    return gmb.lib().gmb_sage_forward_dropout(ctypes.byref(m[0]), x, feats, nodes, ctypes.byref(m[1]), drop(gmb, **d), logits,
                                              ws, ws_bytes, None, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(feats=P, nodes=0), dict(feats=P, nodes=1 << 31), dict(logits=None),
                                 dict(ws=None), dict(ws=P + 8), dict(p=1.5), dict(layer=-1), dict(layer=(1 << 31) - 2),
                                 dict(none=True)], ids=str)
def test_forward_dropout_refuses(gmb, model, bad):
    assert forward(gmb, model, **bad) == EINVAL
    assert gmb.lib().gmb_last_error()


def test_forward_dropout_refuses_a_small_workspace(gmb, model):
    assert forward(gmb, model, ws_bytes=256) == ENOSPC


def backward(gmb, m, x=P, d_logits=P, fws=P, fws_bytes=1 << 40, ws=P, ws_bytes=1 << 40, table=None, nodes=0, grads=True,
             weights=True, **d):
    none = not d
    return gmb.lib().gmb_sage_backward_from(ctypes.byref(m[0]), x, ctypes.byref(m[1]) if weights else None, d_logits,
                                            drop(gmb, none=none, **d), fws, fws_bytes, ctypes.byref(m[2]) if grads else None,
                                            ws, ws_bytes, table, nodes, 0.1, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(d_logits=None), dict(ws=None), dict(ws=P + 8), dict(fws=P + 8),
                                 dict(table=P, nodes=0), dict(table=P + 4, nodes=10), dict(grads=False), dict(weights=False),
                                 dict(p=-0.5), dict(p=0.5, layer=-1), dict(p=0.5, grads=False)], ids=str)
def test_backward_from_refuses(gmb, model, bad):
    assert backward(gmb, model, **bad) == EINVAL
    assert gmb.lib().gmb_last_error()


def test_backward_from_refuses_small_workspaces(gmb, model):
    assert backward(gmb, model, ws_bytes=16) == ENOSPC
    assert backward(gmb, model, fws_bytes=16) == ENOSPC


def test_backward_from_refuses_missing_gradients(gmb, model):
    model[2].d_neigh[0] = None
    assert backward(gmb, model, p=0.5) == EINVAL
