"""Host-only checks of include/symb_block.h: refusals and workspace figures.  No GPU is touched."""
import ctypes as C

import pytest

from paper_2507_03220_amd import binding as sb


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2507_03220_amd import build
    build.build(force=False)


FAKE = 0x1000                                              # aligned, never dereferenced by host-only calls


def _norm(width=64, off=(0, 4), norms=None, kind=0, eps=1e-5, base=0.0):
    return sb.NormBatch(width, off, norms if norms is not None else [sb.Norm(FAKE) for _ in off[1:]], kind, eps, base)


def _norm_status(b):
    out = C.c_size_t(0)
    return sb.lib().symb_norm_workspace_bytes(b.ref(), C.byref(out))


def test_norm_refusals():
    assert _norm_status(_norm()) == sb.SYMB_OK
    assert _norm_status(_norm(off=(0, 0, 0))) == sb.SYMB_OK
    assert _norm_status(_norm(off=(0,))) == sb.SYMB_OK
    for bad in (_norm(width=0), _norm(width=12), _norm(kind=2), _norm(eps=-1.0), _norm(eps=float("nan")), _norm(base=float("inf")), _norm(norms=[sb.Norm(FAKE + 2)]),
                _norm(norms=[sb.Norm(None, None, FAKE + 4)])):
        assert _norm_status(bad) == sb.SYMB_ERR_INVALID_ARG
    assert _norm_status(_norm(off=(0, 4, 3))) == sb.SYMB_ERR_BAD_SEGMENTS
    assert _norm_status(_norm(off=(1, 4))) == sb.SYMB_ERR_BAD_SEGMENTS
    assert _norm_status(_norm(width=sb.SYMB_NORM_MAX_WIDTH + 8)) == sb.SYMB_ERR_UNSUPPORTED
    a, b = FAKE, FAKE + 64
    two = lambda x, y: _norm_status(_norm(off=(0, 2, 4), norms=[sb.Norm(None, None, *x), sb.Norm(None, None, *y)]))  # noqa: E731
    assert two((a, b), (a, b)) == sb.SYMB_OK
    assert two((a, None), (a, None)) == sb.SYMB_OK
    assert two((a, b), (a, None)) == sb.SYMB_ERR_INVALID_ARG       # one of the two alone shared
    assert two((a, b), (b, a)) == sb.SYMB_ERR_INVALID_ARG
    assert two((a, a), (b, None)) == sb.SYMB_ERR_INVALID_ARG       # one buffer for both gradients
    assert sb.lib().symb_norm_workspace_bytes(_norm().ref(), None) == sb.SYMB_ERR_INVALID_ARG
    assert sb.lib().symb_norm_workspace_bytes(None, C.byref(C.c_size_t(0))) == sb.SYMB_ERR_INVALID_ARG


def test_norm_workspace_is_for_gradients_alone():
    assert sb.symb_norm_workspace_bytes(_norm(off=(0, 5000))) == 0
    some = sb.symb_norm_workspace_bytes(_norm(off=(0, 5000), norms=[sb.Norm(None, None, FAKE)]))
    assert some > 0 and some % 256 == 0
    assert sb.symb_norm_workspace_bytes(_norm(off=(0, 0), norms=[sb.Norm(None, None, FAKE)])) == 0


def _kv_status(off=(0, 1), past=(0,), pages=4, N=8, H=2, D=128, P=64, heads=4, window=0):
    b = sb.KvBatch(off, past, None, pages)
    c = sb.symb_kv_cache(FAKE, FAKE, FAKE, FAKE, N, H, D, P)
    out = C.c_size_t(0)
    return sb.lib().symb_kv_workspace_bytes(b.ref(), C.byref(c), heads, window, C.byref(out))


def test_kv_refusals():
    assert _kv_status() == sb.SYMB_OK
    assert _kv_status(past=(255,)) == sb.SYMB_OK
    assert _kv_status(past=(256,)) == sb.SYMB_ERR_INVALID_ARG              # a fifth page
    assert _kv_status(off=(0, 0), past=(10 ** 6,)) == sb.SYMB_OK           # no rows: its pages are not asked for
    assert _kv_status(past=(-1,)) == sb.SYMB_ERR_INVALID_ARG
    assert _kv_status(off=(0, 2, 1), past=(0, 0)) == sb.SYMB_ERR_BAD_SEGMENTS
    for kw in (dict(heads=3), dict(heads=0), dict(heads=-2), dict(window=-1), dict(N=0), dict(H=0), dict(H=-1)):
        assert _kv_status(**kw) == sb.SYMB_ERR_INVALID_ARG, kw
    for kw in (dict(D=96), dict(D=256), dict(P=16), dict(P=48), dict(P=256), dict(pages=(1 << 31) - 1, off=(0, 1, 2), past=(0, 0)),
               dict(past=((1 << 31) - 2,), pages=(1 << 31) - 1), dict(off=(0, (1 << 31) - 1), past=(0,), pages=(1 << 31) - 1)):
        assert _kv_status(**kw) == sb.SYMB_ERR_UNSUPPORTED, kw


def test_a_null_handle_is_refused_and_arguments_are_checked_by_the_binding():
    l = sb.lib()
    b, c = sb.KvBatch([0, 1], [0], None, 4), sb.symb_kv_cache(FAKE, FAKE, FAKE, FAKE, 8, 2, 128, 64)
    assert l.symb_norm_fwd(None, _norm().ref(), FAKE, FAKE, None) == sb.SYMB_ERR_INVALID_ARG
    assert l.symb_norm_bwd(None, _norm().ref(), FAKE, FAKE, FAKE, 0, None, 0, None) == sb.SYMB_ERR_INVALID_ARG
    assert l.symb_kv_append(None, b.ref(), C.byref(c), None, None, 0, 0, None, 0, FAKE, 256, FAKE, 256, None) == sb.SYMB_ERR_INVALID_ARG
    assert l.symb_kv_attention(None, b.ref(), C.byref(c), FAKE, 512, 4, FAKE, 512, 1.0, 0, 0.0, None, 0, None) == sb.SYMB_ERR_INVALID_ARG
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for bad in (x.float(), x[:3], x[:, :32], torch.zeros(64, 4, dtype=torch.bfloat16).t()):
        with pytest.raises(ValueError):
            sb.symb_norm_fwd(None, _norm(), bad, x)
    with pytest.raises(ValueError):
        sb.NormBatch(64, [0, 1], [sb.Norm(torch.zeros(32, dtype=torch.bfloat16))])
    with pytest.raises(ValueError):
        sb.KvBatch([0, 1], [0], torch.zeros(1, 4))
    cache = sb.KvCache.empty(2, 1, 64, 32, device="cpu")
    assert cache.k.shape == (2, 1, 32, 64) and cache.v.shape == (2, 1, 64, 32)
    with pytest.raises(ValueError):
        sb.KvCache(cache.k, cache.k, cache.k_scale, cache.v_scale)
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        sb.symb_kv_attention(None, sb.KvBatch([0, 1], [0], None, 4), cache, q.transpose(1, 2).contiguous().transpose(1, 2), q, 1.0)
