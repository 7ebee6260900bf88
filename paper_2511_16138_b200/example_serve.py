"""A serving step around the store with torch tensors, through the library's public calls.

    python -m paper_2511_16138_b200.example_serve

A long system prompt's keys and values are put into a blob. A batch of requests that begin with it
is probed for the longest stored prefix, the hit chunks are restored once, into pages that all
requests list, and then a layer's decode step runs: the new tokens' keys and values enter the pool
behind the prefix, after norm and rotation (`append_batch`), and their queries attend to what the
pool holds, the common prefix read once for all (`attend_shared_batch`). The script compares with
attention over the plain tensors. Needs a CUDA device and the built library.
"""
from __future__ import annotations

import numpy as np
import torch

from . import lsmkv


def main() -> None:
    dev = torch.device("cuda", 0)
    rng = np.random.default_rng(0)
    g = lsmkv.Geom(n_layers=2, n_kv_heads=8, head_dim=128, page_tokens=16, chunk_tokens=16)
    P, D, H, HQ = g.page_tokens, g.head_dim, g.n_kv_heads, 32
    prefix_pages, n_req = 40, 12
    prefix = rng.integers(0, 32000, prefix_pages * P, dtype=np.uint32)

    def up(a) -> torch.Tensor:
        return torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).reshape(-1).copy()).to(dev)

    def ints(a, kind=torch.int32) -> torch.Tensor:
        return torch.tensor(np.asarray(a, dtype=np.int64), dtype=kind, device=dev)

    def pool(pages):
        return torch.randn(2 * g.n_layers, pages, P, H, D, device=dev).to(torch.bfloat16)

    with lsmkv.Context(g, 0) as ctx:
        # ---- the stored prompt: its pages in one pool, its blob, run and hash index
        src = pool(prefix_pages)
        n = prefix_pages
        keys = torch.empty(n * 32, dtype=torch.uint8, device=dev)
        vals = torch.empty(n * 16, dtype=torch.uint8, device=dev)
        blob = torch.empty(n * g.chunk_bytes, dtype=torch.uint8, device=dev)
        order = rng.permutation(prefix_pages).astype(np.uint32)
        ctx.encode_batch(1, up(prefix), up(np.array([0, len(prefix)], np.uint64)), None,
                         up(np.array([0, n], np.uint64)), n, up(order),
                         lsmkv.pool_table(list(src)), 0, 0, keys, vals, blob, n * g.chunk_bytes)
        run_keys, run_vals = torch.empty_like(keys), torch.empty_like(vals)
        run_n = torch.zeros(1, dtype=torch.int64, device=dev)
        ctx.flush_batch(keys, vals, n, run_keys, run_vals, run_n)
        buckets = lsmkv.lsmkv_hindex_buckets(n)
        hindex = torch.empty(buckets * 32, dtype=torch.uint8, device=dev)
        ctx.hindex_build(run_keys, n, hindex)

        # ---- requests: the prompt and some tokens of their own; one probe finds the prefix
        own = rng.integers(1, 200, n_req)                    # own tokens, the last one being new
        query = np.concatenate([prefix, rng.integers(32000, 64000, P, dtype=np.uint32)])
        q_chunks = len(query) // P
        hit = torch.zeros(1, dtype=torch.int32, device=dev)
        recs = torch.empty(q_chunks * 16, dtype=torch.uint8, device=dev)
        q_off = up(np.array([0, q_chunks], np.uint64))
        ctx.probe_batch(1, up(query), up(np.array([0, len(query)], np.uint64)), q_off, q_chunks,
                        [(run_keys, run_vals, n, None, 0, hindex, buckets)], hit, recs, None)
        assert int(hit.item()) == prefix_pages

        # ---- restored once, into pages that every request's table begins with
        own_pages = -(-own // P)
        num_pages = prefix_pages + int(own_pages.sum()) + 9
        kv = pool(num_pages)                                  # own pages: what earlier steps left
        perm = rng.permutation(num_pages)
        common, rest = perm[:q_chunks], perm[q_chunks:]       # a page for every query chunk
        table = lsmkv.pool_table(list(kv))
        ctx.decode_batch(1, q_off, q_chunks, hit, recs, [(blob, n * g.chunk_bytes)],
                         up(common.astype(np.uint32)), table)
        pages, at = [], 0
        for k in own_pages:
            pages.append(np.concatenate([common[:prefix_pages], rest[at:at + k]]))
            at += k
        kv_len = prefix_pages * P + own
        seqs = lsmkv.Seqs(ints(np.arange(n_req + 1), torch.int64), ints(kv_len),
                          ints(np.cumsum([0] + [len(p) for p in pages]), torch.int64),
                          ints(np.concatenate(pages)), n_new=n_req, max_new=1)
        groups = lsmkv.Groups(ints([0, n_req]), ints([prefix_pages]))

        # ---- a decode step of every layer
        inv = 10000.0 ** (-torch.arange(0, D, 2, device=dev) / D)
        angle = torch.arange(int(kv_len.max()), device=dev)[:, None] * inv
        rope = lsmkv.Rope(torch.cat([angle.cos(), angle.sin()], 1).contiguous())
        norm = (1 + 0.1 * torch.randn(2, D, device=dev)).to(torch.bfloat16)
        scale, worst = D ** -0.5, 0.0
        for layer in range(g.n_layers):
            qkv = torch.randn(n_req, HQ + 2 * H, D, device=dev).to(torch.bfloat16)
            q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:]
            q_turned = torch.empty_like(q)
            out = torch.empty(n_req, HQ, D, dtype=torch.bfloat16, device=dev)
            ctx.append_batch(layer, seqs, k, v, table, rope=rope, q=q, q_out=q_turned,
                             q_norm=norm[0], k_norm=norm[1])
            ctx.attend_shared_batch(layer, seqs, groups, q_turned, out, table, scale)

            # the same over plain tensors
            for i in range(n_req):
                idx = torch.tensor(pages[i].astype(np.int64), device=dev)
                K, V = (kv[b][idx].flatten(0, 1)[:int(kv_len[i])].double().repeat_interleave(HQ // H, 1)
                        for b in (layer, g.n_layers + layer))
                assert torch.equal(kv[layer][idx[:prefix_pages]],
                                   src[layer][torch.tensor(order.astype(np.int64), device=dev)])
                w = torch.softmax(torch.einsum("hd,jhd->hj", q_turned[i].double(), K) * scale, -1)
                want = torch.einsum("hj,jhd->hd", w, V)
                worst = max(worst, float((out[i].double() - want).norm() / want.norm()))
            assert worst < 2 ** -7, worst                     # two roundings to bfloat16
        status = ctx.last_status()
        assert status["flags"] == 0, status
    print("restored %d common pages, %d requests took a step over %d layers, attention within %.1e"
          % (prefix_pages, n_req, g.n_layers, worst))


if __name__ == "__main__":
    main()
