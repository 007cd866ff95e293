"""Refusals of the microscaled store's, product's, model's and distillation's
entry points: bad arguments are found on the host, before anything is
enqueued (addresses here are never read)."""
import ctypes
import os

import pytest

EINVAL, ENOSPC = -1, -2
P = 1 << 40          # an aligned address that nothing reads


@pytest.fixture(scope="module")
def L():
    import paper_2010_05337_amd as gmb
    if not os.path.exists(gmb.LIB_PATH):
        from paper_2010_05337_amd import build
        build.build()
    return gmb.lib()


def test_row_bytes(L):
    for dim, bits, want in [(1, 4, 32), (32, 4, 32), (33, 4, 48), (100, 4, 80), (128, 4, 80), (256, 4, 144),
                            (1, 8, 48), (100, 8, 144), (4096, 4, 2176), (65536, 4, 34816)]:
        assert L.gmb_mx_row_bytes(dim, bits) == want, (dim, bits)
    for dim, bits in [(0, 4), (-1, 4), (65537, 4), (32, 0), (32, 6), (32, 16)]:
        assert L.gmb_mx_row_bytes(dim, bits) == 0
        assert L.gmb_last_error()


def quantise(L, x=P, dtype=0, rs=100, cs=1, ids=None, n_dev=None, n=10, dim=100, fmt=4, table=P, rows=10, stride=80,
             state=None, state_bytes=0):
    return L.gmb_mx_quantise(x, dtype, rs, cs, ids, n_dev, n, dim, fmt, table, rows, stride, state, state_bytes, None,
                             None)


def gather(L, ids=P, n=10, table=P, rows=10, stride=80, dim=100, fmt=4, out=P, dtype=0):
    return L.gmb_mx_gather(ids, None, n, table, rows, stride, dim, fmt, out, dtype, None, None)


def mean(L, indptr=P, ids=P, n=10, table=P, rows=10, stride=80, dim=100, fmt=4, out=P, dtype=0):
    return L.gmb_mx_mean(indptr, ids, None, n, table, rows, stride, dim, fmt, out, dtype, None)


TABLE = [dict(table=None), dict(table=P + 8), dict(rows=0), dict(rows=1 << 31), dict(stride=79), dict(stride=64),
         dict(stride=88), dict(stride=0), dict(stride=-80), dict(dim=0), dict(dim=65537, stride=1 << 20), dict(fmt=5),
         dict(fmt=8), dict(dtype=2), dict(n=-1), dict(n=1 << 31)]


@pytest.mark.parametrize("bad", TABLE + [dict(x=None), dict(n=11), dict(rs=-1), dict(cs=-1), dict(state=P, state_bytes=1 << 20),
                                         dict(ids=P, state=P + 16, state_bytes=1 << 20)], ids=str)
def test_quantise_refuses(L, bad):
    assert quantise(L, **bad) == EINVAL
    assert L.gmb_last_error()


def test_quantise_refuses_a_small_state(L):
    assert quantise(L, ids=P, state=P, state_bytes=256) == ENOSPC


@pytest.mark.parametrize("bad", TABLE + [dict(out=None), dict(ids=None, n=11)], ids=str)
def test_gather_refuses(L, bad):
    assert gather(L, **bad) == EINVAL


@pytest.mark.parametrize("bad", TABLE + [dict(out=None), dict(indptr=None), dict(ids=None)], ids=str)
def test_mean_refuses(L, bad):
    assert mean(L, **bad) == EINVAL


def test_no_rows_enqueue_nothing(L):
    assert quantise(L, n=0, x=None, table=None) == 0
    assert gather(L, n=0, ids=None, table=None, out=None) == 0
    assert mean(L, n=0, indptr=None, table=None) == 0
    assert linear(L, n=0, out=None) == 0


def linear(L, first=None, second=None, n=10, d_in=100, d_out=20, out=P, dtype=0):
    import paper_2010_05337_amd as gmb
    good = dict(rows=P, num_rows=10, row_stride=80, ids=None, weights=P, weight_stride=80)
    a = gmb.MxOperandStruct(**dict(good, **(first or {})))
    b = None if second is None else ctypes.byref(gmb.MxOperandStruct(**dict(good, **second)))
    return L.gmb_mx_linear(ctypes.byref(a), b, None, n, d_in, d_out, None, 0, out, dtype, None, None)


OPERAND = [dict(rows=None), dict(rows=P + 4), dict(num_rows=0), dict(row_stride=72), dict(row_stride=64),
           dict(weights=None), dict(weights=P + 8), dict(weight_stride=16), dict(num_rows=9)]


@pytest.mark.parametrize("bad", OPERAND, ids=str)
def test_linear_refuses_an_operand(L, bad):
    assert linear(L, first=bad) == EINVAL
    assert linear(L, second=bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(second=dict(ids=P)), dict(out=None), dict(n=-1), dict(d_in=0), dict(d_out=0),
                                 dict(d_in=65537), dict(d_out=65537), dict(dtype=4)], ids=str)
def test_linear_refuses(L, bad):
    assert linear(L, **bad) == EINVAL


def test_rows_past_one_launch_are_refused(L):
    # in the product's smallest tiles, a thread for every two rows: 2^32 of them
    n = (1 << 31) - 1
    assert linear(L, first=dict(num_rows=n), n=n, out=None) == EINVAL
    assert b"2^31 - 1024" in L.gmb_last_error()
    b, w = model([(n, n, 1000)], [100, 47])
    assert forward(L, b, w) == EINVAL and L.gmb_mx_forward_workspace_bytes(ctypes.byref(b), ctypes.byref(w)) == 0


def test_linear_refuses_no_operand(L):
    assert L.gmb_mx_linear(None, None, None, 1, 32, 32, None, 0, P, 0, None, None) == EINVAL


def model(caps, dims):
    """Blocks of the capacities (cap_dst, cap_src, cap_nnz) and microscaled
    weights of the widths dims, on addresses that nothing reads."""
    import paper_2010_05337_amd as gmb
    b, w = gmb.BlocksStruct(), gmb.MxWeightsStruct()
    b.num_layers = w.num_layers = len(caps)
    b.num_seeds = caps[-1][0]
    for i, d in enumerate(dims):
        w.dims[i] = d
    for l, (dst, src, nnz) in enumerate(caps):
        k = b.blk[l]
        k.indptr = k.indices = k.nbr = k.src_ids = k.sizes = P
        k.cap_dst, k.cap_src, k.cap_nnz, k.fanout, k.layer = dst, src, nnz, 16, l
        w.w_self[l] = w.w_neigh[l] = w.bias[l] = P
    return b, w


CAPS = [(100, 900, 1000), (10, 100, 90)]


def forward(L, b, w, table=P, rows=1000, stride=80, logits=P, ws=P, ws_bytes=1 << 30):
    return L.gmb_sage_forward_mx(ctypes.byref(b), table, rows, stride, ctypes.byref(w), logits, ws, ws_bytes, None,
                                 None)


def test_model_workspace(L):
    b, w = model(CAPS, [100, 64, 47])
    def up(n):
        return (n + 255) // 256 * 256
    # means of 100 and 64 elements, hidden records of 64
    want = up(100 * 80) + up(100 * 48) + up(10 * 48)
    assert L.gmb_mx_forward_workspace_bytes(ctypes.byref(b), ctypes.byref(w)) == want
    offset = lambda l, hidden: L.gmb_mx_forward_offset(ctypes.byref(b), ctypes.byref(w), l, hidden)  # noqa: E731
    assert [offset(0, 0), offset(0, 1), offset(1, 0)] == [0, up(8000), up(8000) + up(4800)]
    assert offset(1, 1) == offset(-1, 0) == offset(2, 0) == -1


def test_model_refuses(L):
    b, w = model(CAPS, [100, 64, 47])
    assert forward(L, b, w, ws_bytes=100) == ENOSPC
    for bad in (dict(table=None), dict(table=P + 8), dict(rows=0), dict(stride=64), dict(logits=None), dict(ws=None),
                dict(ws=P + 8)):
        assert forward(L, b, w, **bad) == EINVAL, bad
    for name in ("w_self", "w_neigh", "bias"):
        b, w = model(CAPS, [100, 64, 47])
        getattr(w, name)[1] = None
        assert forward(L, b, w) == EINVAL, name
    b, w = model([(100, 900, 1000), (10, 99, 90)], [100, 64, 47])      # block 1's sources are not block 0's rows
    assert forward(L, b, w) == EINVAL
    b, w = model(CAPS, [100, 0, 47])
    assert forward(L, b, w) == EINVAL and L.gmb_mx_forward_workspace_bytes(ctypes.byref(b), ctypes.byref(w)) == 0
    b, w = model(CAPS, [100, 64, 47])
    w.num_layers = 1
    assert forward(L, b, w) == EINVAL
    b, w = model(CAPS, [100, 64, 47])
    b.num_seeds = 0                                                   # an empty batch
    assert forward(L, b, w, logits=None) == 0


def teacher(**over):
    import paper_2010_05337_amd as gmb
    return gmb.TeacherStruct(**dict(dict(logits=P, classes=P, top=4, alpha=0.5, temperature=2.0, reserved=0), **over))


def loss(L, t, logits=P, dtype=0, rows=10, classes=47, out=P, ws=P, ws_bytes=1 << 20, grad=None):
    return L.gmb_distill_loss(logits, dtype, rows, classes, None if t is None else ctypes.byref(t), None, grad, out,
                              ws, ws_bytes, None)


BAD_TEACHERS = [dict(top=0), dict(top=1025), dict(alpha=-0.1), dict(alpha=1.5), dict(alpha=float("nan")),
                dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("inf")),
                dict(temperature=float("nan")), dict(logits=None), dict(classes=None)]


@pytest.mark.parametrize("bad", BAD_TEACHERS, ids=str)
def test_a_bad_teacher_is_refused(L, bad):
    assert loss(L, teacher(**bad)) == EINVAL
    assert backward(L, teacher(**bad)) == EINVAL


def test_distill_refuses(L):
    assert loss(L, None) == EINVAL
    for bad in (dict(logits=None), dict(dtype=3), dict(rows=-1), dict(classes=0), dict(out=None), dict(ws=None),
                dict(ws=P + 4)):
        assert loss(L, teacher(), **bad) == EINVAL, bad
    assert loss(L, teacher(), ws_bytes=16) == ENOSPC
    assert L.gmb_distill_workspace_bytes(10, 47) >= 40
    # rows that workgroups share leave three words each and part
    assert L.gmb_distill_workspace_bytes(1, 131072) > L.gmb_distill_workspace_bytes(1, 47)
    assert L.gmb_distill_workspace_bytes(-1, 47) == 0 and L.gmb_distill_workspace_bytes(10, 0) == 0


@pytest.mark.parametrize("dtype, size", [(0, 4), (1, 2)])
def test_a_gradient_over_the_logits_is_refused(L, dtype, size):
    # (a workspace that is too small is looked at afterwards)
    n = 10 * 47 * size
    for grad, want in ((P, EINVAL), (P + n - size, EINVAL), (P - n + size, EINVAL), (P + n, ENOSPC), (P - n, ENOSPC)):
        assert loss(L, teacher(), dtype=dtype, grad=grad, ws_bytes=16) == want, grad - P


def backward(L, t, dims=(100, 64, 47), table=None, nodes=1000, ws_bytes=1 << 40):
    import paper_2010_05337_amd as gmb
    b, _ = model(CAPS, dims)
    w, g = gmb.WeightsStruct(), gmb.GradsStruct()
    w.num_layers = g.num_layers = 2
    for i, d in enumerate(dims):
        w.dims[i] = d
    for l in range(2):
        w.w_self[l] = w.w_neigh[l] = w.bias[l] = g.d_self[l] = g.d_neigh[l] = g.d_bias[l] = P
    return L.gmb_sage_backward_distill(ctypes.byref(b), P, ctypes.byref(w), P, None if t is None else ctypes.byref(t),
                                       None, P, 1 << 40, ctypes.byref(g), P, P, ws_bytes, table, nodes, 0.1, None)


def test_backward_refuses(L):
    assert backward(L, None) == EINVAL
    assert backward(L, teacher(), dims=(100, 64, 40000)) == EINVAL
    assert backward(L, teacher(), table=P + 4) == EINVAL
    assert backward(L, teacher(), table=P, nodes=0) == EINVAL
    assert backward(L, teacher(), ws_bytes=64) == ENOSPC


def test_the_binding_refuses_host_tensors():
    import torch
    import paper_2010_05337_amd as gmb
    x, rec = torch.zeros(4, 32), torch.zeros(4, 32, dtype=torch.uint8)
    ids = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: gmb.mx_quantise(x, 4), lambda: gmb.mx_gather(ids, rec, 32, 4),
                 lambda: gmb.mx_mean((ids, ids), rec, 32, 4), lambda: gmb.mx_linear(rec, rec, 32),
                 lambda: gmb.distill_loss(x, x, ids.view(4, 1))):
        with pytest.raises(TypeError):
            call()
