"""Sampling several answers to stored prompts on an 8-bit pool, through the library's public calls.

    python -m paper_2511_16138_b200.example_sample

Two prompts' keys and values lie in an 8-bit pool (e4m3 codes, a scale for each block of tokens and
head). They are put into a blob and, on another pool, found and restored by a probe and a get: the
slabs carry their scales along. Each prompt is then forked into several answers (`fork_batch`: whole
pages shared, the begun one copied), which take a few decode steps side by side (`append_batch`,
`attend_batch`); half of them end and give their pages back (`release_batch`), and the pool is
compacted (`compact_pages`), after which the others go on. Every step's result is compared with
attention over the values that the codes stand for. Needs a CUDA device and the built library.
"""
from __future__ import annotations

import numpy as np
import torch

from . import lsmkv


def values(pool, g, buffer, pages):
    """What the codes of some pages of a buffer stand for, [tokens, heads, dim]."""
    P, H, D, B = g.page_tokens, g.n_kv_heads, g.head_dim, g.block_tokens
    slab = pool[buffer][pages]
    x = slab[:, :g.code_bytes].view(torch.float8_e4m3fn).double().unflatten(1, (P // B, B, H, D))
    e = slab[:, g.code_bytes:g.code_bytes + H * (P // B)].double().unflatten(1, (H, P // B)) - 127
    return (x * torch.exp2(e).transpose(1, 2)[:, :, None, :, None]).flatten(0, 2)


def main() -> None:
    dev = torch.device("cuda", 0)
    rng = np.random.default_rng(0)
    gen = torch.Generator(device=dev).manual_seed(0)
    P, D, H, HQ, B, L = 16, 128, 8, 32, 16, 2
    g = lsmkv.Geom(n_layers=L, n_kv_heads=H, head_dim=D, elem_bytes=1, page_tokens=P, chunk_tokens=P,
                   flags=lsmkv.pool_e4m3(B))

    def up(a) -> torch.Tensor:
        return torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).reshape(-1).copy()).to(dev)

    def ints(a, kind=torch.int32) -> torch.Tensor:
        return torch.tensor(np.asarray(a, dtype=np.int64), dtype=kind, device=dev)

    def pool(pages):
        return torch.zeros(2 * L, pages, g.page_bytes, dtype=torch.uint8, device=dev)

    lengths, fan, num_pages = [8 * P, 5 * P], 4, 64
    prompts = [rng.integers(0, 32000, n, dtype=np.uint32) for n in lengths]
    chunks = [n // P for n in lengths]
    n_chunks = sum(chunks)
    with lsmkv.Context(g, 0) as ctx:
        # ---- the prompts' keys and values enter one pool and are put into a blob
        src = pool(n_chunks)
        src_table = lsmkv.pool_table(list(src))
        order = rng.permutation(n_chunks).astype(np.uint32)
        seqs = lsmkv.Seqs(ints(np.cumsum([0] + lengths), torch.int64), ints(lengths),
                          ints(np.cumsum([0] + chunks), torch.int64), ints(order), sum(lengths), max(lengths))
        for layer in range(L):
            k, v = torch.randn(2, sum(lengths), H, D, generator=gen, device=dev).to(torch.bfloat16)
            ctx.append_batch(layer, seqs, k, v, src_table)
        keys = torch.empty(n_chunks * 32, dtype=torch.uint8, device=dev)
        vals = torch.empty(n_chunks * 16, dtype=torch.uint8, device=dev)
        blob = torch.empty(n_chunks * g.chunk_bytes, dtype=torch.uint8, device=dev)
        tokens, off = up(np.concatenate(prompts)), up(np.cumsum([0] + lengths).astype(np.uint64))
        chunk_off = up(np.cumsum([0] + chunks).astype(np.uint64))
        ctx.encode_batch(2, tokens, off, None, chunk_off, n_chunks, up(order), src_table, 0, 0, keys, vals,
                         blob, n_chunks * g.chunk_bytes)
        run_keys, run_vals = torch.empty_like(keys), torch.empty_like(vals)
        run_n = torch.zeros(1, dtype=torch.int64, device=dev)
        ctx.flush_batch(keys, vals, n_chunks, run_keys, run_vals, run_n)

        # ---- another pool: the prompts are found and restored
        kv = pool(num_pages)
        table = lsmkv.pool_table(list(kv))
        refs = torch.zeros(num_pages, dtype=torch.int32, device=dev)
        hit = torch.zeros(2, dtype=torch.int32, device=dev)
        recs = torch.empty(n_chunks * 16, dtype=torch.uint8, device=dev)
        ctx.probe_batch(2, tokens, off, chunk_off, n_chunks, [(run_keys, run_vals, n_chunks)], hit, recs, None)
        assert hit.tolist() == chunks
        places = rng.permutation(num_pages)[:n_chunks].astype(np.uint32)
        ctx.decode_batch(2, chunk_off, n_chunks, hit, recs, [(blob, n_chunks * g.chunk_bytes)], up(places), table)
        assert torch.equal(kv[:, ints(places).long()], src[:, ints(order).long()])
        refs[ints(places).long()] = 1
        # (the last token of each prompt is taken anew, so that its page is a begun one)
        prompt = lsmkv.Tables(ints([n - 1 for n in lengths]), ints(np.cumsum([0] + chunks), torch.int64),
                              ints(places))

        # ---- forked into answers; each has room for two pages more
        parent = ints(np.repeat([0, 1], fan))
        room = np.repeat(chunks, fan) + 2
        answers = lsmkv.Tables(ints(np.zeros(2 * fan)), ints(np.cumsum([0] + list(room)), torch.int64),
                               ints(np.zeros(int(room.sum()))))
        ctx.fork_batch(prompt, parent, answers, refs, table)
        worst, steps = 0.0, 0

        def step(answers, n):
            """One token of every answer in every layer; a page that it needs is the lowest free one."""
            nonlocal worst, steps
            kv_len, page_off, page_table = answers.keep
            length = kv_len.cpu().numpy()
            first, pages = page_off.cpu().numpy(), page_table.cpu().numpy()
            free = iter(np.flatnonzero(refs.cpu().numpy() == 0))
            for i in np.flatnonzero(length % P == 0):
                pages[first[i] + length[i] // P] = page = next(free)
                refs[int(page)] = 1
            page_table.copy_(torch.from_numpy(pages))
            kv_len += 1
            seqs = lsmkv.Seqs(ints(np.arange(n + 1), torch.int64), kv_len, page_off, page_table, n, 1)
            for layer in range(L):
                qkv = torch.randn(n, HQ + 2 * H, D, generator=gen, device=dev).to(torch.bfloat16)
                q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:]
                out = torch.empty(n, HQ, D, dtype=torch.bfloat16, device=dev)
                ctx.append_batch(layer, seqs, k, v, table)
                ctx.attend_batch(layer, seqs, q, out, table, D ** -0.5)
                for i in range(n):
                    idx = torch.from_numpy(pages[first[i]:first[i] + length[i] // P + 1].astype(np.int64)).to(dev)
                    K, V = (values(kv, g, b, idx)[:int(length[i]) + 1].repeat_interleave(HQ // H, 1)
                            for b in (layer, L + layer))
                    w = torch.softmax(torch.einsum("hd,jhd->hj", q[i].double(), K) * D ** -0.5, -1)
                    want = torch.einsum("hj,jhd->hd", w, V)
                    worst = max(worst, float((out[i].double() - want).norm() / want.norm()))
            steps += 1

        for _ in range(P + 3):
            step(answers, 2 * fan)

        # ---- the first half of the answers ends; what is left moves to the pool's beginning
        kv_len, page_off, page_table = answers.keep
        split = int(page_off[fan])
        ctx.release_batch(lsmkv.Tables(kv_len[:fan].clone(), page_off[:fan + 1].clone(), page_table), refs)
        ctx.release_batch(prompt, refs)
        rest = lsmkv.Tables(kv_len[fan:].clone(), (page_off[fan:] - split).contiguous(), page_table[split:].clone())
        used = int((refs > 0).sum())
        live = torch.zeros(1, dtype=torch.int64, device=dev)
        ctx.compact_pages(refs, table, rest.keep[2], n_live=live)
        assert int(live) == used and bool((refs[:used] > 0).all()) and not refs[used:].any()
        for _ in range(3):
            step(rest, fan)
        status = ctx.last_status()
        assert status["flags"] == 0, status
        assert worst < 2 ** -7, worst                         # the roundings of the result and of the weights
    print("restored %d pages, %d answers took %d steps, %d pages in use after compaction, attention within %.1e"
          % (n_chunks, 2 * fan, steps, used, worst))


if __name__ == "__main__":
    main()
