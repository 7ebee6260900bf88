"""8-bit pools through the store's own calls, and the operators on them one after another."""
import numpy as np
import pytest
import torch

from paper_2511_16138_b200 import example_sample, lsmkv
from pool8 import DEV, filled, geom8

pytestmark = pytest.mark.gpu


def test_example(capsys):
    example_sample.main()
    assert "pages in use after compaction" in capsys.readouterr().out


@pytest.mark.parametrize("static", [False, True])
def test_slabs_travel_with_their_scales(static):
    """encode and decode move whole slabs, scales included, with several pages a chunk too."""
    g = lsmkv.Geom(2, 3, 32, elem_bytes=1, page_tokens=8, chunk_tokens=16, flags=lsmkv.pool_e4m3(4))
    assert g.page_bytes == 8 * 3 * 32 + 16 and g.pages_per_chunk == 2
    gen = torch.Generator(device=DEV).manual_seed(1)
    n, num = 5, 40
    src = filled(g, num, gen)
    dst = torch.zeros_like(src)
    rng = np.random.default_rng(0)
    pages, places = rng.permutation(num)[:2 * n], rng.permutation(num)[:2 * n]
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).reshape(-1).copy()).to(DEV)  # noqa: E731
    tokens, off = up(rng.integers(0, 99, n * 16, dtype=np.uint32)), up(np.array([0, n * 16], np.uint64))
    chunk_off = up(np.array([0, n], np.uint64))
    keys, vals = (torch.empty(n * k, dtype=torch.uint8, device=DEV) for k in (32, 16))
    blob = torch.empty(n * g.chunk_bytes, dtype=torch.uint8, device=DEV)
    hit = torch.tensor([n], dtype=torch.int32, device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        ctx.encode_batch(1, tokens, off, None, chunk_off, n, up(pages.astype(np.uint32)),
                         lsmkv.pool_table(list(src)), 0, 0, keys, vals, blob, blob.numel())
        args = (1, chunk_off, n, hit, vals, [(blob, blob.numel())], up(places.astype(np.uint32)),
                lsmkv.pool_table(list(dst)))
        if static:
            lsmkv.lsmkv_decode_batch_static(g, 0, None, *args)
        else:
            ctx.decode_batch(*args)
        assert ctx.last_status()["flags"] == 0
    assert torch.equal(dst[:, torch.tensor(places)], src[:, torch.tensor(pages)])


def test_calls_that_a_pool_does_not_take():
    """A 16-bit dtype's sizes on an 8-bit pool are its own; heads beyond 256 elements are refused."""
    g = geom8(1, 1, 272, 16, 16)
    pool = torch.zeros(2, 2, g.page_bytes, dtype=torch.uint8, device=DEV)
    one = torch.zeros(1, dtype=torch.int32, device=DEV)
    seqs = lsmkv.Seqs(torch.tensor([0, 1], device=DEV), one + 1, torch.tensor([0, 1], device=DEV), one, 1, 1)
    x = torch.zeros(1, 1, 272, dtype=torch.bfloat16, device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        for call in (lambda: ctx.append_batch(0, seqs, x, x, pt), lambda: ctx.attend_batch(0, seqs, x, x, pt, 1.0)):
            with pytest.raises(lsmkv.LsmkvError) as e:
                call()
            assert e.value.code == lsmkv.EINVAL
        with pytest.raises(TypeError):
            ctx.append_batch(0, seqs, x.to(torch.float8_e4m3fn), x.to(torch.float8_e4m3fn), pt)
