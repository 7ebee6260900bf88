"""Undefined queries, keys and values: the rows that see them come out undefined, and no others,
however a row tile is cut among the CTAs, whatever an earlier kernel left behind, and at a cost
that stays near a clean call's.

Tolerances are those of test_attend_gpu.py."""
import math

import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from test_append_gpu import DEV
from test_attend_gpu import check, reference, setup, shared_batch

pytestmark = pytest.mark.gpu


def undefined_exactly(out, lse, ref, lost, dt):
    """Rows (token, head) of `lost` are NaN in every element and in lse, all others as in ref."""
    assert torch.isnan(out[lost]).all() and torch.isnan(lse[lost]).all()
    o, A, want_lse, sub = ref
    check(out[~lost], lse[~lost], (o[~lost], A[~lost], want_lse[~lost], sub[~lost]), dt)


QUERIES = [
    # dtype, D, P, hq, hkv, new, history
    (torch.bfloat16, 128, 16, 32, 8, [1] * 8, [1000, 300, 40, 0, 2000, 700, 128, 129]),   # cut tiles
    (torch.float16, 64, 16, 8, 8, [1] * 200, [5, 20, 130, 0] * 50),                       # mostly whole
    (torch.bfloat16, 256, 16, 8, 2, [1, 2, 1], [900, 300, 20]),
    (torch.bfloat16, 128, 16, 8, 2, [3, 2, 4], [1500, 40, 700]),                          # several tokens
    (torch.bfloat16, 128, 16, 8, 2, [70, 300], [900, 2000]),                              # many rows, cut
    (torch.float16, 64, 16, 16, 16, [200, 257] * 12, [0, 1] * 12),                        # many rows, whole
    (torch.bfloat16, 96, 5, 6, 2, [90], [400]),
]


@pytest.mark.parametrize("case", QUERIES, ids=[str(i) for i in range(len(QUERIES))])
def test_undefined_queries_give_undefined_rows(case):
    dt, D, P, hq = case[:4]
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    lost.view(-1)[1::3] = True
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    q[lost] = math.nan
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
        assert ctx.last_status()["flags"] == 0
    undefined_exactly(out, lse, ref, lost, dt)


# The key is alone in its tile of 128 keys for the rows that see no later one. 59 sequences of two KV
# heads and nine key tiles: spans of 148 CTAs begin right before the ninth tile in every fourth.
KEYS = [
    (torch.bfloat16, 128, 16, 8, 2, [1] * 59, [1024] * 59, 1024),
    (torch.float16, 64, 16, 4, 2, [1] * 59, [1024] * 59, 1024),
    (torch.bfloat16, 128, 16, 8, 2, [3] * 59, [1023] * 59, 1024),
    (torch.bfloat16, 128, 16, 8, 2, [40] * 59, [1004] * 59, 1024),
    (torch.float16, 64, 16, 8, 2, [150] * 40, [1004] * 40, 1024),
]


@pytest.mark.parametrize("case", KEYS, ids=[str(i) for i in range(len(KEYS))])
def test_a_lone_undefined_key_reaches_the_rows_that_see_it(case):
    dt, D, P, hq, hkv, new, hist, key = case
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case[:7], n_layers=1)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    for i in range(len(new)):
        pool[0, int(table[page_off[i] + key // P]), key % P] = math.nan
        lost[new_off[i] + max(0, key - hist[i]):new_off[i + 1]] = True
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
        assert ctx.last_status()["flags"] == 0
    undefined_exactly(out, lse, ref, lost, dt)


PREFIXES = [
    # as SHARED of test_attend_gpu.py: 65 common pages are eight key tiles and 16 keys
    (torch.bfloat16, 128, 16, 32, 8, [8], [65], 1, (0, 40)),                # few rows
    (torch.bfloat16, 128, 16, 8, 2, [2] * 59, [65] * 59, 1, (0, 40)),       # many rows
    (torch.float16, 64, 16, 8, 2, [2] * 59, [65] * 59, 3, (0, 300)),
]


@pytest.mark.parametrize("what", ["queries", "keys"])
@pytest.mark.parametrize("case", PREFIXES, ids=[str(i) for i in range(len(PREFIXES))])
def test_undefined_rows_over_shared_prefixes(case, what):
    dt, D, P = case[:3]
    geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(case)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    if what == "queries":
        lost.view(-1)[1::3] = True
        q[lost] = math.nan
    else:
        members, pages = case[5], case[6]
        first = 0
        for g, n in enumerate(members):
            if g % 3 != 1:                                  # the last common page of the group
                pool[0, int(table[page_off[first] + pages[g] - 1])] = math.nan
                lost[new_off[first]:new_off[first + n]] = True
            first += n
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_shared_batch(0, seqs, groups, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
        assert ctx.last_status()["flags"] == 0
    undefined_exactly(out, lse, ref, lost, dt)


@pytest.mark.parametrize("D", [80, 96])
def test_what_an_earlier_kernel_left_on_chip_does_not_matter(D):
    """A call whose sums are all NaN, then one with narrower heads over long histories, every wait
    limited to about a millisecond: nothing of the first shows in the second, in time either."""
    case = (torch.bfloat16, 128, 16, 32, 8, [2048], [0])
    geom, pool, q, seqs, *_ = setup(case, n_layers=1)
    pool[1] = math.nan
    with lsmkv.Context(geom, 0) as ctx:
        out = torch.zeros_like(q)
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08)
        assert ctx.last_status()["flags"] == 0 and torch.isnan(out).all()
    case = (torch.bfloat16, D, 16, 8, 2, [100] * 100, [20000] + [900] * 99)
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.1)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.set_tuning("wait_cycles", 2_000_000)
        out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.1, lse)
        assert ctx.last_status()["flags"] == 0
    check(out, lse, ref, torch.bfloat16)
