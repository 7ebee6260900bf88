"""Release, fork, compaction and page copies against a plain restatement on the host; every result is equal
bit for bit."""
import numpy as np
import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from pool8 import geom8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a, d=torch.int32):
    return torch.tensor(np.asarray(a, dtype=np.int64), dtype=d, device=DEV)


def host(t):
    return t.cpu().numpy().astype(np.int64) & 0xFFFFFFFF


def geom(kind, L=3, H=2, D=16, P=8, B=4):
    return geom8(L, H, D, P, B) if kind == 8 else lsmkv.Geom(L, H, D, page_tokens=P, chunk_tokens=P)


def random_pool(g, num, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, 256, (2 * g.n_layers, num, g.page_bytes), generator=gen, device=DEV, dtype=torch.uint8)


def fork_model(g, kv, off, table, parent, kid_off, kid_table, refs, pool):
    """(kid_len, kid_table, refs, pool) after a fork, children in order."""
    P, row = g.page_tokens, g.code_bytes // g.page_tokens
    kid_table, refs, pool = kid_table.copy(), refs.copy(), pool.copy()
    before = refs.copy()
    free = iter(np.flatnonzero(before == 0))
    kid_len = []
    for c, i in enumerate(parent):
        pages = table[off[i]:off[i] + -(-kv[i] // P)]
        kid_len.append(kv[i])
        tail = kv[i] % P
        mine = pages.copy()
        if tail:
            mine[-1] = next(free, 0xFFFFFFFF)
            if mine[-1] != 0xFFFFFFFF:
                n = -(-tail * row // 16) * 16
                pool[:, mine[-1], :n] = pool[:, pages[-1], :n]
                pool[:, mine[-1], g.code_bytes:] = pool[:, pages[-1], g.code_bytes:]
        for p in mine:
            if p != 0xFFFFFFFF:
                refs[p] += 1
        kid_table[kid_off[c]:kid_off[c] + len(mine)] = mine
    return np.array(kid_len), kid_table, refs, pool


def sequences(rng, n, P, most, num):
    kv = rng.integers(0, most + 1, n)
    counts = -(-kv // P)
    off = np.cumsum([0] + [int(c) + int(rng.integers(0, 3)) for c in counts])
    table = np.full(off[-1], 0xFFFFFFFF, dtype=np.int64)
    perm, at = rng.permutation(num), 0
    refs = np.zeros(num, dtype=np.int64)
    for i in range(n):
        table[off[i]:off[i] + counts[i]] = perm[at:at + counts[i]]
        refs[perm[at:at + counts[i]]] += 1
        at += counts[i]
    return kv, off, table, refs


def signed(a):
    return np.where(a > 0x7FFFFFFF, a - (1 << 32), a)


@pytest.mark.parametrize("kind", [8, 16])
@pytest.mark.parametrize("n,fan,most,num", [(1, 1, 1, 4), (1, 7, 20, 40), (5, 3, 100, 200), (40, 9, 60, 9000),
                                            (3, 700, 50, 20000), (2, 4, 4000, 30000)])
def test_fork_equals_the_model_and_release_undoes_it(kind, n, fan, most, num):
    rng = np.random.default_rng(n * fan + most)
    g = geom(kind, L=1 if num > 500 else 3)
    kv, off, table, refs = sequences(rng, n, g.page_tokens, most, num)
    kv[0] = max(kv[0], 0)
    parent = rng.integers(0, n, n * fan)
    room = -(-kv[parent] // g.page_tokens) + rng.integers(0, 2, n * fan)
    kid_off = np.cumsum([0] + list(room))
    kid_table = np.full(kid_off[-1], 7, dtype=np.int64)
    pool = random_pool(g, num)
    want = fork_model(g, kv, off, table, parent, kid_off, kid_table, refs, pool.cpu().numpy())
    tables = lsmkv.Tables(dev(kv), dev(off, torch.int64), dev(signed(table)))
    kids = lsmkv.Tables(dev(np.full(n * fan, 99)), dev(kid_off, torch.int64), dev(kid_table))
    r = dev(refs)
    with lsmkv.Context(g, 0) as ctx:
        ctx.fork_batch(tables, dev(parent), kids, r, lsmkv.pool_table(list(pool)))
        assert ctx.last_status()["flags"] == 0
        assert np.array_equal(host(kids.keep[0]), want[0])
        assert np.array_equal(host(kids.keep[2]), want[1])
        assert np.array_equal(host(r), want[2])
        assert np.array_equal(pool.cpu().numpy(), want[3])
        assert np.array_equal(host(tables.keep[2]), table & 0xFFFFFFFF) and np.array_equal(host(tables.keep[0]), kv)
        ctx.release_batch(kids, r)
        assert ctx.last_status()["flags"] == 0
        assert np.array_equal(host(r), refs)
        ctx.release_batch(tables, r)
        assert ctx.last_status()["flags"] == 0 and not r.any()
        # nothing left to give back
        ctx.release_batch(tables, r)
        st = ctx.last_status()
        if (kv > 0).any():
            assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == int(np.flatnonzero(kv > 0)[0])
        assert not r.any()


def test_fork_without_free_pages_and_with_bad_children():
    g = geom(16)
    P = g.page_tokens
    kv = [2 * P + 3, P]
    table = np.array([4, 1, 7, 2])
    refs = np.zeros(9, dtype=np.int64)
    refs[[4, 1, 7, 2]] = 1
    refs[[0, 3, 5]] = 2                                    # free: 6 and 8
    parent = [0, 1, 0, 5, 0, 0]                            # child 3: no such parent; child 4: no room
    kid_off = np.cumsum([0, 3, 1, 3, 3, 2, 3])
    pool = random_pool(g, 9)
    before = pool.cpu().numpy()
    tables = lsmkv.Tables(dev(kv), dev([0, 3, 4], torch.int64), dev(table))
    kids = lsmkv.Tables(dev([50] * 6), dev(kid_off, torch.int64), dev([70] * 15))
    r = dev(refs)
    with lsmkv.Context(g, 0) as ctx:
        ctx.fork_batch(tables, dev(parent), kids, r, lsmkv.pool_table(list(pool)))
        st = ctx.last_status()
    assert st["flags"] == lsmkv.ST_BAD_COUNT | lsmkv.ST_NO_PAGE and st["first_bad"] == 3
    assert host(kids.keep[2]).tolist() == [4, 1, 6, 2, 4, 1, 8] + [70] * 5 + [4, 1, 0xFFFFFFFF]
    assert host(kids.keep[0]).tolist() == [kv[0], kv[1], kv[0], 50, 50, kv[0]]
    refs[[4, 1]] += 3
    refs[2] += 1
    refs[[6, 8]] = 1
    assert np.array_equal(host(r), refs)
    n = 3 * g.code_bytes // P
    before[:, [6, 8], :n] = before[:, [7], :n]
    assert np.array_equal(pool.cpu().numpy(), before)


def test_bad_pages_are_reported():
    g = geom(16)
    P = g.page_tokens
    pool = random_pool(g, 6)
    before = pool.clone()
    tables = lsmkv.Tables(dev([2 * P + 1, P]), dev([0, 3, 4], torch.int64), dev([0, 40, 41, 5]))
    kids = lsmkv.Tables(dev([0]), dev([0, 3], torch.int64), dev([9, 9, 9]))
    r = dev([1, 0, 0, 0, 0, 1])
    with lsmkv.Context(g, 0) as ctx:
        ctx.fork_batch(tables, dev([0]), kids, r, lsmkv.pool_table(list(pool)))
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == 1
        assert host(kids.keep[2]).tolist() == [0, 40, 41] and host(r).tolist() == [2, 0, 0, 0, 0, 1]
        assert torch.equal(pool, before)
        ctx.release_batch(tables, r)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == 1
        assert host(r).tolist() == [1, 0, 0, 0, 0, 0]
        # a sequence longer than its entries, and entries beyond the table
        for kv, off, item in (([2 * P, P], [0, 1, 2], 0), ([P, P], [0, 1, 9], 1)):
            t = lsmkv.Tables(dev(kv), dev(off, torch.int64), dev([0, 5]))
            r = dev([3, 0, 0, 0, 0, 3])
            ctx.release_batch(t, r)
            st = ctx.last_status()
            assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == item
            assert host(r).tolist() == [[3, 0, 0, 0, 0, 2], [2, 0, 0, 0, 0, 3]][item]
        ctx.copy_pages(dev([0, 1, 2]), dev([3, 6, 4]), lsmkv.pool_table(list(pool)))
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == 1
        before[:, 3], before[:, 4] = before[:, 0], before[:, 2]
        assert torch.equal(pool, before)
        table, refs = dev([0, 77, 5, 5]), dev([1, 0, 0, 0, 0, 2])
        ctx.compact_pages(refs, lsmkv.pool_table(list(pool)), table)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == 1
        assert host(table).tolist() == [0, 77, 1, 1] and host(refs).tolist() == [1, 2, 0, 0, 0, 0]


@pytest.mark.parametrize("kind", [8, 16])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("num,live", [(1, 0.0), (1, 1.0), (30, 0.5), (1000, 0.1), (1000, 1.0), (1000, 0.0),
                                      (9000, 0.7), (30001, 0.4)])
def test_compaction_equals_the_model(kind, in_place, num, live):
    rng = np.random.default_rng(num)
    g = geom(kind, L=1 if num > 500 else 3)
    refs = np.where(rng.random(num) < live, rng.integers(1, 5, num), 0)
    table = rng.permutation(np.repeat(np.arange(num), refs))
    pool = random_pool(g, num)
    want = pool.cpu().numpy()
    n = int((refs > 0).sum())
    src, dst = n + np.flatnonzero(refs[n:]), np.flatnonzero(refs[:n] == 0)
    place = np.arange(num)
    place[src] = dst
    want[:, dst] = want[:, src]
    want_refs = refs.copy()
    want_refs[dst], want_refs[src] = refs[src], 0
    r, t = dev(refs), dev(table)
    r_out, t_out = (r, t) if in_place else (torch.full_like(r, 77), torch.full_like(t, 77))
    live_out = torch.full((1,), -5, dtype=torch.int64, device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        ctx.compact_pages(r, lsmkv.pool_table(list(pool)), t, refs_out=r_out, table_out=t_out, n_live=live_out)
        assert ctx.last_status()["flags"] == 0
        assert int(live_out) == n
        assert np.array_equal(host(r_out), want_refs) and np.array_equal(host(t_out), place[table])
        assert np.array_equal(pool.cpu().numpy()[:, :n], want[:, :n])
        # compact already: nothing moves
        again = pool.clone()
        ctx.compact_pages(r_out, lsmkv.pool_table(list(pool)), t_out)
        assert ctx.last_status()["flags"] == 0
        assert np.array_equal(host(r_out), want_refs) and np.array_equal(host(t_out), place[table])
        assert torch.equal(pool, again)


def test_copies_of_pages_larger_than_a_stage():
    g = lsmkv.Geom(2, 8, 128, page_tokens=32, chunk_tokens=32)             # 64 KiB a slab
    pool = random_pool(g, 50)
    want = pool.clone()
    rng = np.random.default_rng(1)
    perm = rng.permutation(50)
    src, dst = perm[:20], perm[20:40]
    want[:, dev(dst).long()] = pool[:, dev(src).long()]
    with lsmkv.Context(g, 0) as ctx:
        ctx.set_tuning("copy_stage_bytes", 4096 + 16)
        ctx.copy_pages(dev(src), dev(dst), lsmkv.pool_table(list(pool)))
        assert ctx.last_status()["flags"] == 0
        assert torch.equal(pool, want)
        ctx.copy_pages(dev(src), dev(src), lsmkv.pool_table(list(pool)))
        assert torch.equal(pool, want)


def test_captured_fork_and_compaction_replay():
    g = geom(8)
    P = g.page_tokens
    rng = np.random.default_rng(3)
    kv, off, table, refs = sequences(rng, 6, P, 90, 300)
    parent = np.repeat(np.arange(6), 3)
    kid_off = np.cumsum([0] + [-(-kv[i] // P) for i in parent])
    pool = random_pool(g, 300)
    pt = lsmkv.pool_table(list(pool))
    tables = lsmkv.Tables(dev(kv), dev(off, torch.int64), dev(signed(table)))
    kids = lsmkv.Tables(dev([0] * 18), dev(kid_off, torch.int64), dev(np.zeros(kid_off[-1])))
    r, r_out, t_out = dev(refs), dev(refs), torch.zeros_like(kids.keep[2])
    par = dev(parent)
    with lsmkv.Context(g, 0) as ctx:
        def step():
            ctx.fork_batch(tables, par, kids, r, pt)
            ctx.compact_pages(r, pt, kids.keep[2], refs_out=r_out, table_out=t_out)

        state = pool.clone()
        step()
        torch.cuda.synchronize()
        first = [x.clone() for x in (kids.keep[0], kids.keep[2], r, r_out, t_out, pool)]
        graph = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
            step()
        ctx.compact_pages(torch.zeros(100000, dtype=torch.int32, device=DEV), (pt[0], 100000),
                          t_out[:0])                                       # larger scratch; no page is used
        for _ in range(3):
            r.copy_(dev(refs))
            pool.copy_(state)
            graph.replay()
            torch.cuda.synchronize()
            for x, y in zip((kids.keep[0], kids.keep[2], r, r_out, t_out, pool), first):
                assert torch.equal(x, y)
        assert ctx.last_status()["flags"] == 0


def test_a_wait_that_runs_out_is_reported():
    """No copy is started for one piece: its wait runs out after the limit, the call ends and says so."""
    g = geom(16)
    pool = random_pool(g, 8)
    with lsmkv.Context(g, 0) as ctx:
        ctx.set_tuning("wait_cycles", 1000000)
        ctx.set_tuning("test_drop_piece", 0)
        ctx.copy_pages(dev([0, 1]), dev([4, 5]), lsmkv.pool_table(list(pool)))
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_WAIT_EXPIRED and st["first_bad"] == 0
        ctx.set_tuning("test_drop_piece", -1)
        ctx.copy_pages(dev([0, 1]), dev([4, 5]), lsmkv.pool_table(list(pool)))
        assert ctx.last_status()["flags"] == 0
        assert torch.equal(pool[:, 4:6], pool[:, :2])


def test_refusals():
    g = geom(16)
    pool = random_pool(g, 8)
    pt = lsmkv.pool_table(list(pool))
    t = lsmkv.Tables(dev([3]), dev([0, 1], torch.int64), dev([0]))
    r = dev([1] * 8)
    with lsmkv.Context(g, 0) as ctx:
        for call in (lambda: ctx.fork_batch(t, dev([0]), t, r, (0, 8)),
                     lambda: ctx.copy_pages(dev([0]), dev([1]), (0, 8)),
                     lambda: ctx.compact_pages(r, (0, 8), dev([0]))):
            with pytest.raises(lsmkv.LsmkvError) as e:
                call()
            assert e.value.code == lsmkv.EINVAL
        for call in (lambda: ctx.fork_batch(t, dev([0, 0]), t, r, pt), lambda: ctx.fork_batch(t, dev([0]), t, r[:5], pt),
                     lambda: ctx.compact_pages(r[:5], pt, dev([0])), lambda: ctx.copy_pages(dev([0]), dev([1, 2]), pt),
                     lambda: ctx.compact_pages(r, pt, dev([0]), table_out=dev([0, 0])),
                     lambda: ctx.compact_pages(r, pt, dev([0]), n_live=dev([0])),
                     lambda: ctx.release_batch(t, r.long()), lambda: ctx.release_batch(t, r.cpu())):
            with pytest.raises(ValueError):
                call()
        # empty calls
        ctx.copy_pages(dev([]), dev([]), pt)
        none = lsmkv.Tables(dev([]), dev([0], torch.int64), dev([]))
        ctx.release_batch(none, r)
        ctx.fork_batch(t, dev([]), none, r, pt)
        assert ctx.last_status()["flags"] == 0 and host(r).tolist() == [1] * 8
