"""Append and attend calls without a GPU: struct layouts of the binding, refusals that need no
device, and the binding's own checks of shapes and types."""
import ctypes

import pytest
import torch

from paper_2511_16138_b200 import lsmkv


def z(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype)


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(lsmkv.SeqsStruct) == 48
    assert ctypes.sizeof(lsmkv.RopeStruct) == 32
    assert ctypes.sizeof(lsmkv.GroupsStruct) == 24
    # lsmkv_rows_t (24 bytes) after another, then lsmkv_pool_t (16 bytes)
    a, b = lsmkv._AttendArgs, lsmkv._AppendArgs
    assert (a.q.offset, a.out.offset, a.kv_ptrs.offset) == (0, a.OUT, a.POOL) == (0, 24, 48)
    assert ctypes.sizeof(a) == 64 and ctypes.sizeof(b) == 112
    assert (b.k.offset, b.v.offset, b.q.offset, b.out.offset, b.kv_ptrs.offset) == \
        (0, b.V, b.Q, b.OUT, b.POOL) == (0, 24, 48, 72, 96)


def test_calls_without_a_context_are_refused():
    L = lsmkv.lib()
    seqs = lsmkv.SeqsStruct(1, 1, 1)
    ref = ctypes.addressof(seqs)
    assert L.lsmkv_append_batch(None, None, 0, 0, ref, None, None, None, None, 0, None, None, None,
                                None, 1e-6) == lsmkv.EINVAL
    assert L.lsmkv_attend_batch(None, None, 0, 0, ref, 1, None, None, 1.0, None, None) == lsmkv.EINVAL
    assert L.lsmkv_attend_shared_batch(None, None, 0, 0, ref, None, 1, None, None, 1.0, None,
                                       None) == lsmkv.EINVAL


def test_the_batch_descriptors_check_their_tensors():
    ok = dict(new_off=z(3, dtype=torch.int64), kv_len=z(2), page_off=z(3, dtype=torch.int64),
              page_table=z(5), n_new=2, max_new=1)
    s = lsmkv.Seqs(**ok)
    assert (s.c.n_new, s.c.n_seq, s.c.max_new) == (2, 2, 1)
    assert s.c.kv_len == ok["kv_len"].data_ptr()
    for bad in (dict(new_off=z(3)), dict(new_off=z(2, dtype=torch.int64)), dict(kv_len=z(4)[::2]),
                dict(page_off=z(4, dtype=torch.int64)), dict(page_table=z(5, dtype=torch.int64))):
        with pytest.raises(ValueError):
            lsmkv.Seqs(**(ok | bad))
    assert lsmkv.Groups(z(3), z(2)).c.n_group == 2
    for a, b in ((z(2), z(2)), (z(3, dtype=torch.int64), z(2)), (z(6)[::2], z(2))):
        with pytest.raises(ValueError):
            lsmkv.Groups(a, b)
    table = torch.zeros(7, 64)
    r = lsmkv.Rope(table, True, z(4))
    assert (r.c.n_pos, r.c.rot_dim, r.c.interleaved, r.n_positions) == (7, 64, 1, 4)
    for a, b in ((table.double(), None), (table[:, ::2], None), (table, z(4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            lsmkv.Rope(a, positions=b)


def test_rows_and_types_are_checked():
    t = torch.zeros(4, 6, 16, dtype=torch.bfloat16)
    assert lsmkv._rows("q", t, 4, 6, 16) == (t.data_ptr(), 96, 16)
    assert lsmkv._rows("q", t[:, 2:4], 4, 2, 16) == (t.data_ptr() + 64, 96, 16)
    for n, heads, dim in ((3, 6, 16), (4, 5, 16), (4, 6, 8)):
        with pytest.raises(ValueError):
            lsmkv._rows("q", t, n, heads, dim)
    with pytest.raises(ValueError):
        lsmkv._rows("q", t[..., ::2], 4, 6, 8)
    assert lsmkv._dtype(t, None, t) == lsmkv.BF16 and lsmkv._dtype(t.half()) == lsmkv.F16
    for other in (t.half(), t.float()):
        with pytest.raises(TypeError):
            lsmkv._dtype(t, other)
    with pytest.raises(TypeError):
        lsmkv._dtype(t.float())


def test_the_stride_of_an_extent_of_one_does_not_matter():
    wide = torch.zeros(3, 5 * 16 + 3, dtype=torch.bfloat16)
    one = wide.as_strided((1, 4, 16), (83, 16, 1))                  # a token of a row of 83 elements
    assert lsmkv._rows("q", one, 1, 4, 16) == (one.data_ptr(), 64, 16)
    head = torch.zeros(4, 16, dtype=torch.bfloat16).as_strided((4, 1, 16), (16, 3, 1))
    assert lsmkv._rows("k", head, 4, 1, 16) == (head.data_ptr(), 16, 16)
    both = wide[:1, :16].as_strided((1, 1, 16), (83, 5, 1))
    assert lsmkv._rows("k", both, 1, 1, 16) == (both.data_ptr(), 16, 16)


class OnDevice(torch.Tensor):
    """A host tensor that says it lies on the device: stands in for one here."""
    is_cuda = True


def device(t):
    return t.as_subclass(OnDevice)


def test_tensors_in_host_memory_are_refused_before_the_call():
    ctx = lsmkv.Context.__new__(lsmkv.Context)          # no device here: a handle that every call refuses
    ctx.handle, ctx.geom = None, lsmkv.Geom(1, 2, 16)

    def seqs(where=device):
        return lsmkv.Seqs(where(z(2, dtype=torch.int64)), where(z(1)), where(z(2, dtype=torch.int64)),
                          where(z(1)), 1, 1)

    def groups(where=device):
        return lsmkv.Groups(where(z(2)), where(z(1)))

    host = lambda t: t  # noqa: E731
    rows = lambda heads, where=device: where(torch.zeros(1, heads, 16, dtype=torch.bfloat16))  # noqa: E731
    pool = (device(z(2, dtype=torch.int64)), 1)
    good = dict(layer=0, seqs=seqs(), q=rows(4), out=rows(4), pool=pool, scale=1.0, stream=0)
    bad = [dict(seqs=seqs(host)), dict(q=rows(4, host)), dict(out=rows(4, host)),
           dict(pool=(z(2, dtype=torch.int64), 1)), dict(lse=torch.zeros(1, 4))]
    for change, error in [({}, lsmkv.LsmkvError)] + [(b, ValueError) for b in bad]:
        with pytest.raises(error):
            ctx.attend_batch(**(good | change))
        with pytest.raises(error):
            ctx.attend_shared_batch(groups=groups(), **(good | change))
    with pytest.raises(ValueError):
        ctx.attend_shared_batch(groups=groups(host), **good)
    good = dict(layer=0, seqs=seqs(), k=rows(2), v=rows(2), pool=pool, q=rows(4), stream=0,
                rope=lsmkv.Rope(device(torch.zeros(3, 16))))
    weights = torch.zeros(16, dtype=torch.bfloat16)
    for change, error in ({}, lsmkv.LsmkvError), (dict(pool=(0, 1)), lsmkv.LsmkvError), \
            (dict(seqs=seqs(host)), ValueError), (dict(k=rows(2, host)), ValueError), \
            (dict(v=rows(2, host)), ValueError), (dict(q=rows(4, host)), ValueError), \
            (dict(q_out=rows(4, host)), ValueError), (dict(q_norm=weights), ValueError), \
            (dict(k_norm=weights), ValueError), (dict(rope=lsmkv.Rope(torch.zeros(3, 16))), ValueError):
        with pytest.raises(error):
            ctx.append_batch(**(good | change))
