"""8-bit pools and page calls without a GPU: geometry, struct layouts, refusals that need no device."""
import ctypes

import pytest
import torch

from paper_2511_16138_b200 import lsmkv


def z(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype)


def test_geometry_of_8_bit_pools():
    g = lsmkv.Geom(4, 8, 128, elem_bytes=1, page_tokens=16, chunk_tokens=32, flags=lsmkv.pool_e4m3(16))
    assert g.block_tokens == 16 and g.code_bytes == 16 * 8 * 128 and g.page_bytes == g.code_bytes + 16
    assert g.chunk_bytes == 2 * 2 * 4 * g.page_bytes
    one = lsmkv.Geom(4, 3, 48, elem_bytes=1, page_tokens=24, chunk_tokens=24, flags=lsmkv.pool_e4m3(1))
    assert one.page_bytes == 24 * 3 * 48 + 80                       # 72 scales in whole 16 bytes
    plain = lsmkv.Geom(4, 8, 128)
    assert plain.block_tokens == 0 and plain.page_bytes == plain.code_bytes


def test_geometries_that_are_refused():
    """Refused before any device is looked for."""
    ok = dict(n_layers=2, n_kv_heads=4, head_dim=64, elem_bytes=1, page_tokens=16, chunk_tokens=16,
              flags=lsmkv.pool_e4m3(16))
    for bad in (dict(elem_bytes=2), dict(head_dim=72), dict(page_tokens=24, chunk_tokens=24), dict(flags=lsmkv.pool_e4m3(0)),
                dict(flags=lsmkv.pool_e4m3(3)), dict(flags=lsmkv.pool_e4m3(32)), dict(flags=lsmkv.pool_e4m3(4) | 1),
                dict(flags=4), dict(flags=lsmkv.pool_e4m3(4) | 1 << 16), dict(flags=0x400)):
        with pytest.raises(lsmkv.LsmkvError) as e:
            lsmkv.lsmkv_create(lsmkv.Geom(**(ok | bad)))
        assert e.value.code == lsmkv.EINVAL


def test_struct_layouts_match_the_header():
    t = lsmkv.TablesStruct
    assert ctypes.sizeof(t) == 40
    assert (t.n_entries.offset, t.n_seq.offset, t.kv_len.offset, t.page_off.offset, t.page_table.offset) == \
        (0, 8, 16, 24, 32)


def test_calls_without_a_context_are_refused():
    L = lsmkv.lib()
    t = lsmkv.TablesStruct(1, 1)
    ref, p = ctypes.addressof(t), lsmkv.PoolStruct(None, 4)
    assert L.lsmkv_release_batch(None, None, ref, None, 4) == lsmkv.EINVAL
    assert L.lsmkv_fork_batch(None, None, ref, None, ref, None, ctypes.byref(p)) == lsmkv.EINVAL
    assert L.lsmkv_compact_pages(None, None, None, None, None, None, 0, ctypes.byref(p), None) == lsmkv.EINVAL
    assert L.lsmkv_copy_pages(None, None, None, None, 1, ctypes.byref(p)) == lsmkv.EINVAL


def test_tables_check_their_tensors():
    ok = dict(kv_len=z(2), page_off=z(3, dtype=torch.int64), page_table=z(5))
    t = lsmkv.Tables(**ok)
    assert (t.c.n_seq, t.c.n_entries, t.n_seq) == (2, 5, 2) and t.c.kv_len == ok["kv_len"].data_ptr()
    for bad in (dict(kv_len=z(4)[::2]), dict(kv_len=z(2, dtype=torch.int64)), dict(page_off=z(3)),
                dict(page_off=z(4, dtype=torch.int64)), dict(page_table=z(5, dtype=torch.int64))):
        with pytest.raises(ValueError):
            lsmkv.Tables(**(ok | bad))


def test_tensors_in_host_memory_are_refused():
    ctx = lsmkv.Context.__new__(lsmkv.Context)
    ctx.handle, ctx.geom = None, lsmkv.Geom(1, 2, 16)
    t = lsmkv.Tables(z(1), z(2, dtype=torch.int64), z(1))
    for call in (lambda: ctx.release_batch(t, z(4)), lambda: ctx.fork_batch(t, z(1), t, z(4), (1, 4)),
                 lambda: ctx.copy_pages(z(1), z(1), (1, 4)), lambda: ctx.compact_pages(z(4), (1, 4), z(1))):
        with pytest.raises(ValueError):
            call()
