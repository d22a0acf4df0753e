"""Host-only checks of include/symb_loss.h: refusals and workspace figures.  No GPU is touched."""
import ctypes as C

import pytest
import torch

from paper_2507_03220_amd import binding as sb


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2507_03220_amd import build
    build.build(force=False)


def _batch(width=64, vocab=100, off=(0, 4), losses=None, reduction=0, cap=0.0):
    return sb.LossBatch(width, vocab, off, losses if losses is not None else [sb.Loss() for _ in off[1:]], reduction, cap)


def _status(b, entries=0, gradient=1):
    out = C.c_size_t(0)
    return sb.lib().symb_loss_workspace_bytes(b.ref(), entries, gradient, C.byref(out))


def test_refusals():
    assert _status(_batch()) == _status(_batch(), 5) == _status(_batch(vocab=1)) == _status(_batch(off=(0, 0, 0))) == _status(_batch(off=(0,))) == sb.SYMB_OK
    nan, inf = float("nan"), float("inf")
    for bad in (_batch(width=0), _batch(width=-8), _batch(width=12), _batch(vocab=0), _batch(vocab=-1), _batch(reduction=2), _batch(reduction=-1), _batch(cap=-1.0), _batch(cap=nan),
                _batch(cap=inf), _batch(losses=[sb.Loss(nan)]), _batch(losses=[sb.Loss(inf)])):
        assert _status(bad) == sb.SYMB_ERR_INVALID_ARG
    for t in (0.0, -1.0, nan, inf):
        assert _status(_batch(losses=[sb.Loss(1.0, t)])) == sb.SYMB_OK                  # (cross entropy does not look at it)
        assert _status(_batch(losses=[sb.Loss(1.0, t)]), 3) == sb.SYMB_ERR_INVALID_ARG
    for t in (2.0 ** -20, 2.0 ** 20):
        assert _status(_batch(losses=[sb.Loss(1.0, t)]), 3) == sb.SYMB_OK
    for t in (2.0 ** -21, 1e-39, 2.0 ** 21):
        assert _status(_batch(losses=[sb.Loss(1.0, t)]), 3) == sb.SYMB_ERR_UNSUPPORTED
    assert _status(_batch(), -1) == sb.SYMB_ERR_INVALID_ARG
    for off in ((0, 4, 3), (1, 4)):
        assert _status(_batch(off=off)) == sb.SYMB_ERR_BAD_SEGMENTS
    assert _status(_batch(), sb.SYMB_LOSS_MAX_ENTRIES) == _status(_batch(vocab=sb.SYMB_LOSS_MAX_VOCAB)) == _status(_batch(width=sb.SYMB_LOSS_MAX_WIDTH)) == sb.SYMB_OK
    assert _status(_batch(), sb.SYMB_LOSS_MAX_ENTRIES + 1) == _status(_batch(vocab=sb.SYMB_LOSS_MAX_VOCAB + 1)) == _status(_batch(width=sb.SYMB_LOSS_MAX_WIDTH + 8)) == sb.SYMB_ERR_UNSUPPORTED
    assert _status(_batch(width=4096, off=(0, 2 ** 19 - 1))) == sb.SYMB_OK
    assert _status(_batch(width=4096, off=(0, 2 ** 19))) == sb.SYMB_ERR_UNSUPPORTED        # 2^31 elements of X
    assert _status(_batch(width=8, off=(0, sb.SYMB_LOSS_MAX_ROWS))) == sb.SYMB_OK
    assert _status(_batch(width=8, off=(0, sb.SYMB_LOSS_MAX_ROWS + 1))) == sb.SYMB_ERR_UNSUPPORTED
    assert _status(_batch(off=tuple(range(180001)))) == sb.SYMB_ERR_UNSUPPORTED            # descriptors: 2 MiB at most
    assert _status(_batch(off=tuple(range(170001)))) == sb.SYMB_OK
    assert sb.lib().symb_loss_workspace_bytes(_batch().ref(), 0, 1, None) == sb.SYMB_ERR_INVALID_ARG
    assert sb.lib().symb_loss_workspace_bytes(None, 0, 1, C.byref(C.c_size_t(0))) == sb.SYMB_ERR_INVALID_ARG
    assert sb.lib().symb_cross_entropy(None, _batch().ref(), *[None] * 7, 0, None) == sb.SYMB_ERR_INVALID_ARG
    assert sb.lib().symb_distillation(None, _batch().ref(), *[None] * 4, 1, *[None] * 4, 0, None) == sb.SYMB_ERR_INVALID_ARG
    assert sb.lib().symb_distillation(None, _batch().ref(), *[None] * 4, 0, *[None] * 4, 0, None) == sb.SYMB_ERR_INVALID_ARG


def test_workspace_is_bounded():
    """It holds the weights of some rows, not the logits of all."""
    assert sb.symb_loss_workspace_bytes(_batch(off=(0, 0))) == 0
    for rows in (1, 300, 8192, 100000):
        n = sb.symb_loss_workspace_bytes(_batch(4608, 256000, (0, rows)))
        assert 0 < n < 3 << 30 and n % 256 == 0
        assert sb.symb_loss_workspace_bytes(_batch(4608, 256000, (0, rows)), gradient=False) < 300 << 20
    assert sb.symb_loss_workspace_bytes(_batch(4608, 256000, (0, 8192))) < 8192 * 256000 * 4 // 3


def test_the_binding_looks_at_its_tensors():
    b, bf, i32, f32 = _batch(), torch.bfloat16, torch.int32, torch.float32
    X, W, y = torch.zeros(4, 64, dtype=bf), torch.zeros(100, 64, dtype=bf), torch.zeros(4, dtype=i32)
    good = dict(X=X, W=W, labels=y, loss=torch.zeros(1), row_loss=torch.zeros(4), dX=torch.zeros(4, 64, dtype=bf))
    for name, bad in (("X", X.float()), ("X", X[:3]), ("X", torch.zeros(4, 128, dtype=bf)[:, ::2]), ("W", W.t().contiguous()), ("W", W[:99]), ("labels", y.long()), ("labels", y[:3]),
                      ("loss", torch.zeros(2)), ("loss", torch.zeros(1, dtype=torch.float64)), ("row_loss", torch.zeros(5)), ("dX", torch.zeros(4, 64))):
        with pytest.raises(ValueError):
            sb.symb_cross_entropy(None, b, **{**good, name: bad})
    del good["labels"]
    ids, logits = torch.zeros(4, 6, dtype=i32), torch.zeros(4, 6, dtype=f32)
    for a, c in ((ids.long(), logits), (ids, logits.to(bf)), (ids[:, :5], logits), (ids[:3], logits[:3]), (ids[0], logits[0]), (torch.zeros(6, 4, dtype=i32).t(), logits)):
        with pytest.raises(ValueError):
            sb.symb_distillation(None, b, good["X"], good["W"], a, c, good["loss"])
    with pytest.raises(ValueError):
        sb.LossBatch(64, 100, (0, 4, 5), [sb.Loss()])
