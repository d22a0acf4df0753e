"""What a call's descriptors have room for (one slot of 2 MiB, include/symb_block.h): the workspace queries refuse what the calls refuse.  No GPU is touched but by the last test."""
import ctypes as C

import pytest

from paper_2507_03220_amd import binding as sb


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2507_03220_amd import build
    build.build(force=False)


FAKE = 0x1000
SLOT = 2 << 20


def _kv(tokens, group, window=0, P=128, past=0):
    b, c, out = sb.KvBatch([0, tokens], [past], None, -(-(tokens + past) // P)), sb.symb_kv_cache(FAKE, FAKE, FAKE, FAKE, 1, 1, 128, P), C.c_size_t(0)
    return sb.lib().symb_kv_workspace_bytes(b.ref(), C.byref(c), group, window, C.byref(out))


def test_attention_work_items():
    """Tiles of 128 rows at 32 bytes each: 65536 of them fill the slot, the rest of it being a few empty lists."""
    assert _kv(170000, 48) == sb.SYMB_OK
    assert _kv(175000, 48) == sb.SYMB_ERR_UNSUPPORTED
    assert _kv(128 * 65530, 1) == sb.SYMB_OK
    assert _kv(128 * 65536, 1) == sb.SYMB_ERR_UNSUPPORTED
    assert _kv((1 << 31) - 2000, 1, past=100) == sb.SYMB_ERR_UNSUPPORTED          # (at once: no list of sixteen million items is made first)
    text = sb.lib().symb_last_error(None).decode()
    assert "work items" in text, text


def test_norm_descriptors():
    """32 bytes a segment, 16 a chunk of rows and 24 a gradient: 29000 segments of a row each fit, 29200 do not."""
    def status(S):
        b, out = sb.NormBatch(8, range(S + 1), [sb.Norm(None, None, FAKE + 64 * i) for i in range(S)]), C.c_size_t(0)
        return sb.lib().symb_norm_workspace_bytes(b.ref(), C.byref(out))
    assert (32 + 16 + 24) * 29000 < SLOT < (32 + 16 + 24) * 29200
    assert status(29000) == sb.SYMB_OK
    assert status(29200) == sb.SYMB_ERR_UNSUPPORTED


@pytest.mark.gpu
def test_the_calls_refuse_the_same():
    import torch

    import gpu_harness as gh
    cache = sb.KvCache.empty(4, 1, 128, 128)
    q = torch.zeros(175000, 48, 128, device="cuda", dtype=torch.bfloat16)
    table = torch.zeros(1, 1368, device="cuda", dtype=torch.int32)
    with pytest.raises(sb.SymbError) as e:
        sb.symb_kv_attention(gh.handle(), sb.KvBatch([0, 175000], [0], table), cache, q, q, 1.0, ws=q, stream=gh.stream_ptr())
    assert e.value.status == sb.SYMB_ERR_UNSUPPORTED and "work items" in str(e.value)
    # an append's pages: 16 bytes each
    T = 32 * (SLOT // 16 + 1)
    k = torch.zeros(T, 1, 64, device="cuda", dtype=torch.bfloat16)
    small = sb.KvCache.empty(4, 1, 64, 32)
    with pytest.raises(sb.SymbError) as e:
        sb.symb_kv_append(gh.handle(), sb.KvBatch([0, T], [0], torch.full((1, T // 32), -1, device="cuda", dtype=torch.int32)), small, None, None, None, k, k, gh.stream_ptr())
    assert e.value.status == sb.SYMB_ERR_UNSUPPORTED and "pages" in str(e.value)
    S = 29200
    g, x = torch.empty(S, 8, device="cuda"), torch.zeros(S, 8, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(sb.SymbError) as e:
        sb.symb_norm_bwd(gh.handle(), sb.NormBatch(8, range(S + 1), [sb.Norm(None, None, g[i].data_ptr()) for i in range(S)]), x, x, x, 0, torch.empty(1 << 21, device="cuda"), gh.stream_ptr())
    assert e.value.status == sb.SYMB_ERR_UNSUPPORTED
    torch.cuda.synchronize()
