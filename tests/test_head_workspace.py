"""The workspace of the cross-entropy over many classes is bounded for any number
of rows and classes together (sizes are asked for on the host; nothing is
allocated or launched)."""
import os

import pytest

P = 1 << 40          # an aligned address that nothing reads
MB = 1 << 20


@pytest.fixture(scope="module")
def gmb():
    import paper_2010_05337_amd as gmb
    if not os.path.exists(gmb.LIB_PATH):
        from paper_2010_05337_amd import build
        build.build()
    gmb.lib()
    return gmb


def up(x, to):
    return -(-x // to) * to


def bound(n, d, classes, dtype, aligned):
    """Copies of x (fp32: two, of two parts) and of W, 384 MB of gradients of
    logits (256 classes of them at least), sums of a piece of the classes: dW's
    at most 128 MB, dx's 64 MB and twice its size, dbias's a 64th of the
    gradients' number; the rows' statistics."""
    es = 1 if dtype else 2
    pad_n, pad_d = up(n, 256), up(d, 64)
    copies = pad_n * pad_d * 2 * es * es + (0 if dtype and aligned else classes * pad_d * 2 * es)
    grads = max(384 * MB, pad_n * 256 * 2 * es) + pad_n * 256 * 2 * es
    stats = 8 * (512 * 256 + 3 * pad_n) + 32 * pad_n + MB
    return copies + grads + 128 * MB + 64 * MB + 2 * n * up(d, 4) * 4 + grads // 32 + stats


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("turned", [0, 1])
@pytest.mark.parametrize("n, d, classes", [
    (16_384, 256, 2_449_029), (45_000, 256, 2_449_029), (100_000, 256, 1_000_000), (1000, 128, 100_000_000), (4000, 256, 100_000),
    (1 << 22, 64, 100_000), (4097, 8, 1 << 27), (300, 1024, 1_000_000), (40, 2000, 500_000), (70_000, 65, 4_000_003)], ids=str)
def test_the_workspace_is_bounded(gmb, n, d, classes, dtype, turned):
    head = gmb.LinearHeadStruct(P, d, P, 1 if turned else d, classes if turned else 1, P, P, n, d, classes, dtype, 0)
    need = gmb.lib().gmb_linear_loss_workspace_bytes(head, gmb.LinearGradsStruct(P, P, P, turned, 0))
    most = bound(n, d, classes, dtype, d % 64 == 0 and not turned)
    assert 0 < need <= most, (need / MB, most / MB)
    alone = gmb.lib().gmb_linear_loss_workspace_bytes(head, None)
    assert 0 < alone < need
