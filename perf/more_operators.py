"""Cases of the operators on 8-bit pools and of the page calls: append and attend where the pool
holds 8-bit floats (e4m3) with a power-of-two scale for each block of tokens and head; fork (with the
release of the generation before) and compaction of a pool's pages.

Sizes follow this repository's workloads: the Llama-3-8B KV shape (32 layers, 8 KV heads of 128, pages
of 16, 256 requests of 1k to 8k tokens), the small-head GQA shape (28 layers, 4 KV heads, pages of 64,
512 conversations, turns of 256 to 1024 tokens) and the long-context shape (8 KV heads under 64 query
heads, requests of 32768 tokens whose last 1k changed).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E_MIN, E_MAX = -100, 100          # exponents of a block's scale
_contexts = {}


# ---- cases -------------------------------------------------------------------------------

def _step(name, op, dtype, hq, hkv, dim, page, block, n_seq, new, hist, shape_seed=1, norm=False,
          rot=0, interleaved=False):
    c = {"op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "dim": dim, "page": page, "block": block,
         "n_seq": n_seq, "new_lo": new[0], "new_hi": new[1], "hist_lo": hist[0],
         "hist_hi": hist[1], "shape_seed": shape_seed}
    if op == "append":
        c.update(norm=norm, rot=rot or dim, interleaved=interleaved)
    if name:
        c["name"] = name
    return c


def _fork(name, layers, hkv, dim, page, block, n_seq, fan, hist, spare, shape_seed=1):
    c = {"op": "fork", "layers": layers, "hkv": hkv, "dim": dim, "page": page, "block": block,
         "n_seq": n_seq, "fan": fan, "hist_lo": hist[0], "hist_hi": hist[1], "spare": spare,
         "shape_seed": shape_seed}
    return dict(c, name=name) if name else c


def _compact(name, layers, hkv, dim, page, block, n_page, live, shape_seed=1):
    c = {"op": "compact", "layers": layers, "hkv": hkv, "dim": dim, "page": page, "block": block,
         "n_page": n_page, "live": live, "shape_seed": shape_seed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of a lightly loaded server: latency counts
        _step("append8_step_8", "append", "bf16", 32, 8, 128, 16, 16, 8, (1, 1), (100, 1000)),
        # a full decode step of a model that normalises queries and keys per head
        _step("append8_step_512_norm", "append", "fp16", 28, 4, 128, 64, 16, 512, (1, 1),
              (64, 1024), norm=True),
        # the next turn of 64 conversations enters the cache
        _step("append8_turn", "append", "bf16", 28, 4, 128, 64, 16, 64, (256, 1024), (0, 2048),
              norm=True),
        # a decode step of four short chats: latency counts
        _step("attend8_step_4", "attend", "bf16", 32, 8, 128, 16, 16, 4, (1, 1), (200, 1000)),
        # a decode step of the Llama-3-8B-shaped workload
        _step("attend8_step_llama8b", "attend", "bf16", 32, 8, 128, 16, 16, 256, (1, 1),
              (1023, 8191)),
        # a decode step of 512 conversations on four KV heads, a scale for every token
        _step("attend8_step_gqa4", "attend", "fp16", 28, 4, 128, 64, 1, 512, (1, 1), (256, 4096)),
        # what is left of 32 prompts after their stored prefixes were restored, from one token on
        _step("attend8_suffix", "attend", "bf16", 32, 8, 128, 16, 16, 32, (1, 512), (512, 4096)),
        # two long-context requests whose last 1k tokens changed
        _step("attend8_long", "attend", "bf16", 64, 8, 128, 16, 16, 2, (1024, 1024),
              (31744, 31744)),
        # one prompt sampled eight ways: latency counts
        _fork("fork_8", 32, 8, 128, 16, 0, 1, 8, (1000, 1000), 64),
        # 64 prompts continued four ways each, all layers
        _fork("fork_64x4", 32, 8, 128, 16, 0, 64, 4, (100, 1000), 300),
        # a small 8-bit pool after a few requests have left
        _compact("compact8_small", 28, 4, 128, 64, 16, 300, 0.5),
        # a pool of which two in five pages were given back
        _compact("compact_large", 32, 8, 128, 16, 0, 1000, 0.6),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng: random.Random):
    op = rng.choice(("append", "attend", "attend", "fork", "compact"))
    hq, hkv = rng.choice(((32, 8), (28, 4), (64, 8), (16, 16), (24, 4), (16, 2), (40, 8)))
    dim = rng.choice((64, 96, 128, 128))
    page = rng.choice((16, 16, 32, 64))
    block = rng.choice((1, 4, 8, 16, 16))
    dtype = rng.choice(("bf16", "fp16"))
    seed = rng.randrange(1, 1 << 30)
    if op == "append":
        n_seq = _log(rng, 1, 512)
        hi = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, min(4096, 40000 // n_seq)))
        return _step(None, op, dtype, hq, hkv, dim, page, block, n_seq, (1, hi),
                     (0, _log(rng, 8, 1024)), seed, norm=rng.random() < 0.5,
                     rot=rng.choice((dim, dim, dim // 2)), interleaved=rng.random() < 0.3)
    if op == "attend":
        if rng.random() < 0.5:                                        # one token each
            n_seq = _log(rng, 1, 512)
            hi = _log(rng, 16, max(16, min(65536, 1000000 // n_seq)))
            return _step(None, op, dtype, hq, hkv, dim, page, block, n_seq, (1, 1), (hi // 5, hi),
                         seed)
        n_seq = _log(rng, 1, 32)                                      # a suffix or a prompt
        new = _log(rng, 2, 2048)
        hist = _log(rng, 1, 16384)
        while n_seq > 1 and n_seq * hq * new * (new + hist) > 4e9:
            n_seq //= 2
        while n_seq * hq * new * (new + hist) > 4e9:
            new = (new + 1) // 2
        return _step(None, op, dtype, hq, hkv, dim, page, block, n_seq, (1, new),
                     (hist // 3, hist), seed)
    layers = rng.choice((4, 28, 32))
    block = rng.choice((0, block))
    slab = 2 * layers * page * hkv * dim * (2 - bool(block))          # bytes of a page
    if op == "fork":
        pages = max(24, int(2e9) // slab)
        fan = _log(rng, 2, 16)
        n_seq = _log(rng, 1, max(1, min(64, pages // (4 * fan))))
        hist = max(2, min(2048, pages // 2 // n_seq * page))
        return _fork(None, layers, hkv, dim, page, block, n_seq, fan, (hist // 4, hist),
                     rng.randint(8, max(8, pages // 4)), seed)
    return _compact(None, layers, hkv, dim, page, block, _log(rng, 24, max(24, int(2e9) // slab)),
                    round(rng.uniform(0.2, 0.9), 2), seed)


# ---- lengths and page tables -------------------------------------------------------------

def _cum(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


def _shape(case):
    """new and kv of every sequence: the case's own."""
    r = random.Random(case["shape_seed"])
    n = case["n_seq"]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    return new, [a + r.randint(case["hist_lo"], case["hist_hi"]) for a in new]


def _fork_shape(case):
    r = random.Random(case["shape_seed"])
    return [r.randint(max(1, case["hist_lo"]), max(1, case["hist_hi"])) for _ in range(case["n_seq"])]


def _live(case):
    """References to every page of a pool to be compacted."""
    r = random.Random(case["shape_seed"])
    return [(1 if r.random() < 0.8 else r.randint(2, 8)) if r.random() < case["live"] else 0
            for _ in range(case["n_page"])]


def _row_bytes(case):
    """Bytes of a page of one layer's keys: codes or 16-bit floats, and scales in whole 16 bytes."""
    body = case["page"] * case["hkv"] * case["dim"]
    if not case["block"]:
        return 2 * body, 2 * body
    return body, body + -(-case["hkv"] * (case["page"] // case["block"]) // 16) * 16


def work(case):
    if case["op"] == "compact":
        refs = _live(case)
        n = sum(1 for x in refs if x)
        moves = sum(1 for x in refs[n:] if x)
        return {"bytes": 2 * moves * 2 * case["layers"] * _row_bytes(case)[1] + 8 * len(refs)
                + 8 * sum(refs), "flops": 0}
    if case["op"] == "fork":
        body, page = _row_bytes(case)
        rows, entries = 0, 0
        for n in _fork_shape(case):
            r = n % case["page"]
            rows += case["fan"] * (r * (body // case["page"]) + (page - body if r else 0))
            entries += case["fan"] * -(-n // case["page"])
        # the copies; table entries read and written; counters down and up
        return {"bytes": 2 * rows * 2 * case["layers"] + 4 * entries * 7, "flops": 0}
    new, kv = _shape(case)
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    t = sum(new)
    if case["op"] == "append":
        rows = t * (2 * hq + 2 * hkv) * d * 2 + t * 2 * hkv * d            # read, q written; codes
        scales = 2 * hkv * sum(-(-b // case["block"]) - (b - a) // case["block"]
                               for a, b in zip(new, kv))
        flops = 6 * t * (hq + hkv) * case["rot"] / 2 + 3 * t * 2 * hkv * d
        if case["norm"]:
            flops += 4 * t * (hq + hkv) * d
        return {"bytes": rows + scales + t * case["rot"] * 4 + 4 * t, "flops": flops}
    seen = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(new, kv))
    read = sum(kv)
    return {"bytes": 2 * read * hkv * d + 2 * hkv * (read // case["block"]) + 2 * t * hq * d * 2
            + 4 * (read // case["page"]), "flops": 4 * seen * hq * d}


# ---- inputs ------------------------------------------------------------------------------

def _exponent(amax):
    """Least e with amax <= 448 * 2^e, within the scale's range; 448 = 1.75 * 2^8."""
    bits = amax.float().contiguous().view(torch.int32)
    return ((bits + 0x1FFFFF) >> 23).sub_(135).clamp_(E_MIN, E_MAX)


def _power(e):
    """2^e in 32 bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _views(buf, P, hkv, d, block):
    """Codes [pages, P, hkv, d] and scales [pages, hkv, P / block] of a pool's 8-bit buffer."""
    body = P * hkv * d
    codes = buf[:, :body].view(torch.float8_e4m3fn).unflatten(1, (P, hkv, d))
    scales = buf[:, body:body + hkv * (P // block)].unflatten(1, (hkv, P // block))
    return codes, scales


def _fill(buf, P, hkv, d, block, normal, spread):
    """Quantised values in every page, as earlier steps leave them."""
    codes, scales = _views(buf, P, hkv, d, block)
    some = max(1, (1 << 26) // (P * hkv * d))
    for a in range(0, buf.shape[0], some):
        n = min(some, buf.shape[0] - a)
        x = normal(n, P // block, block, hkv, d).float().mul_(spread)
        e = _exponent(x.abs().amax((2, 4)))                           # [n, blocks, hkv]
        x.mul_(_power(-e)[:, :, None, :, None])
        codes[a:a + n] = x.flatten(1, 2).to(torch.float8_e4m3fn)
        scales[a:a + n] = (e + 127).transpose(1, 2).to(torch.uint8)


def _geom(case, lsmkv, layers):
    flags = lsmkv.pool_e4m3(case["block"]) if case["block"] else 0
    return lsmkv.Geom(n_layers=layers, n_kv_heads=case["hkv"], head_dim=case["dim"],
                      elem_bytes=1 if case["block"] else 2, page_tokens=case["page"],
                      chunk_tokens=case["page"], flags=flags)


def _context(geom, lsmkv):
    if geom not in _contexts:
        _contexts[geom] = lsmkv.Context(geom, torch.cuda.current_device())
    return _contexts[geom]


def _generator(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + case["shape_seed"])
    return g


def _pages_pool(case, g, num_pages):
    """All layers' buffers of a pool [2 L, pages, bytes], as numbers of two bytes or one."""
    size = (2 * case["layers"], num_pages, _row_bytes(case)[1] // (1 if case["block"] else 2))
    if case["block"]:
        return torch.randint(0, 256, size, generator=g, device=DEV, dtype=torch.uint8)
    return torch.randn(size, generator=g, device=DEV, dtype=torch.bfloat16).view(torch.int16)


def _prepare_fork(case, seed):
    g = _generator(case, seed)
    P, fan, kv = case["page"], case["fan"], _fork_shape(case)
    pages = [-(-n // P) for n in kv]
    kids = [i for i in range(len(kv)) for _ in range(fan)]
    kid_pages = [pages[i] for i in kids]
    partial = [1 if kv[i] % P else 0 for i in kids]
    num_pages = sum(pages) + sum(partial) + case["spare"]
    perm = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)
    off, kid_off = _cum(pages), _cum(kid_pages)
    table = perm[:off[-1]].contiguous()
    # the generation before: children of the same prompts, with pages of their own at the end
    owner = torch.repeat_interleave(torch.arange(len(kids)), torch.tensor(kid_pages))
    local = torch.arange(kid_off[-1]) - torch.tensor(kid_off)[owner]
    source = torch.tensor(off)[torch.tensor(kids)[owner]] + local
    kid_table = table[source.to(DEV)]
    last = torch.tensor([kid_off[c + 1] - 1 for c in range(len(kids)) if partial[c]], dtype=torch.int64)
    kid_table[last.to(DEV)] = perm[off[-1]:off[-1] + len(last)]
    refs = torch.zeros(num_pages, dtype=torch.int32, device=DEV)
    one = torch.ones((), dtype=torch.int32, device=DEV)
    refs.index_put_((table.long(),), one, accumulate=True)
    refs.index_put_((kid_table.long(),), one, accumulate=True)
    s = {"case": dict(case), "op": "fork", "refs": refs, "num_pages": num_pages,
         "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
         "page_off": torch.tensor(off, device=DEV), "page_table": table,
         "parent": torch.tensor(kids, dtype=torch.int32, device=DEV),
         "kid_len": torch.tensor([kv[i] for i in kids], dtype=torch.int32, device=DEV),
         "kid_off": torch.tensor(kid_off, device=DEV), "kid_table": kid_table,
         "pool_data": _pages_pool(case, g, num_pages)}
    s["pool"] = (torch.tensor([b.data_ptr() for b in s["pool_data"]], device=DEV), num_pages)
    if own:
        from paper_2511_16138_b200 import lsmkv
        s["ctx"] = _context(_geom(case, lsmkv, case["layers"]), lsmkv)
        s["tables"] = lsmkv.Tables(s["kv_len"], s["page_off"], s["page_table"])
        s["kids"] = lsmkv.Tables(s["kid_len"], s["kid_off"], s["kid_table"])
    return s


def _prepare_compact(case, seed):
    g = _generator(case, seed)
    refs = torch.tensor(_live(case), dtype=torch.int32, device=DEV)
    # every reference is an entry of some sequence's table, in random order
    table = torch.repeat_interleave(torch.arange(case["n_page"], device=DEV), refs.long())
    table = table[torch.randperm(len(table), generator=g, device=DEV)].to(torch.int32)
    s = {"case": dict(case), "op": "compact", "refs": refs, "page_table": table,
         "refs_out": torch.empty_like(refs), "table_out": torch.empty_like(table),
         "n_live": torch.zeros(1, dtype=torch.int64, device=DEV),
         "pool_data": _pages_pool(case, g, case["n_page"])}
    s["pool"] = (torch.tensor([b.data_ptr() for b in s["pool_data"]], device=DEV), case["n_page"])
    if own:
        from paper_2511_16138_b200 import lsmkv
        s["ctx"] = _context(_geom(case, lsmkv, case["layers"]), lsmkv)
    return s


def prepare(case, seed):
    if case["op"] == "fork":
        return _prepare_fork(case, seed)
    if case["op"] == "compact":
        return _prepare_compact(case, seed)
    new, kv = _shape(case)
    dt, g = DTYPES[case["dtype"]], _generator(case, seed)
    P, hq, hkv, d, block = (case[k] for k in ("page", "hq", "hkv", "dim", "block"))

    def normal(*shape, scale=1.0):
        x = torch.randn(shape, generator=g, device=DEV, dtype=dt)
        return x if scale == 1.0 else x.mul_(scale)

    # a fragmented pool: pages in random order
    pages = [-(-b // P) for b in kv]
    page_off = _cum(pages)
    num_pages = page_off[-1] + 8
    perm = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)
    s = {
        "case": dict(case), "op": case["op"], "scale": d ** -0.5,
        "n_new": sum(new), "max_new": max(new), "max_kv": max(kv),
        "new_off": torch.tensor(_cum(new), device=DEV),
        "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
        "page_off": torch.tensor(page_off, device=DEV),
        "page_table": perm[:page_off[-1]].contiguous(),
    }
    # the elements of a key head differ in size, as a trained model's do
    spread = (0.4 * torch.randn(hkv, d, generator=g, device=DEV)).exp()
    for name, by in (("K", spread), ("V", torch.ones_like(spread))):
        buf = torch.zeros(num_pages, _row_bytes(case)[1], dtype=torch.uint8, device=DEV)
        _fill(buf, P, hkv, d, block, normal, by)
        s[name], (s[name + "c"], s[name + "s"]) = buf, _views(buf, P, hkv, d, block)
    s["pool"] = (torch.tensor([s["K"].data_ptr(), s["V"].data_ptr()], device=DEV), num_pages)
    if case["op"] == "append":
        # what the projection of a layer leaves: q, k and v of a token side by side
        qkv = normal(sum(new), hq + 2 * hkv, d)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["k"].mul_(spread)
        s["out"] = torch.empty(sum(new), hq, d, dtype=dt, device=DEV)
        rot = case["rot"]
        inv = 500000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
        ang = torch.arange(max(kv), device=DEV, dtype=torch.float64)[:, None] * inv
        s["table"] = torch.cat([ang.cos(), ang.sin()], 1).float()
        s["q_norm"] = s["k_norm"] = None
        if case["norm"]:
            s["q_norm"], s["k_norm"] = 1 + normal(d, scale=0.1), 1 + normal(d, scale=0.1)
    else:
        # queries long enough that scores spread as a trained model's do
        s["q"] = normal(sum(new), hq, d, scale=2.0)
        s["out"] = torch.empty_like(s["q"])
    if own:
        # the handle and the step's descriptors, which a serving loop keeps over all its layers
        from paper_2511_16138_b200 import lsmkv
        s["ctx"] = _context(_geom(case, lsmkv, 1), lsmkv)
        s["seqs"] = lsmkv.Seqs(s["new_off"], s["kv_len"], s["page_off"], s["page_table"],
                               s["n_new"], s["max_new"])
        if case["op"] == "append":
            s["rope"] = lsmkv.Rope(s["table"], interleaved=case["interleaved"])
    return s


# ---- the operators -----------------------------------------------------------------------

def run(s):
    if s["op"] == "append":
        if own:
            s["ctx"].append_batch(0, s["seqs"], s["k"], s["v"], s["pool"], rope=s["rope"],
                                  q=s["q"], q_out=s["out"], q_norm=s["q_norm"],
                                  k_norm=s["k_norm"], eps=1e-6)
        q = s["out"] if own else _plain_append(s)
        return q, s["Kc"], s["Ks"].view(torch.float8_e8m0fnu), s["Vc"], \
            s["Vs"].view(torch.float8_e8m0fnu)
    if s["op"] == "attend":
        if own:
            s["ctx"].attend_batch(0, s["seqs"], s["q"], s["out"], s["pool"], s["scale"])
            return s["out"]
        return _plain_attend(s)
    if s["op"] == "fork":
        # a generation's pages are given back and the next one takes its own
        if own:
            s["ctx"].release_batch(s["kids"], s["refs"])
            s["ctx"].fork_batch(s["tables"], s["parent"], s["kids"], s["refs"], s["pool"])
        else:
            _plain_fork(s)
        return s["kid_table"], s["refs"], s["pool_data"]
    if own:
        s["ctx"].compact_pages(s["refs"], s["pool"], s["page_table"], refs_out=s["refs_out"],
                               table_out=s["table_out"], n_live=s["n_live"])
    else:
        _plain_compact(s)
    return s["table_out"], s["refs_out"], s["n_live"], s["pool_data"]


def _rows(s):
    """Sequence and position of every new token."""
    t = torch.arange(s["n_new"], device=DEV)
    seq = torch.searchsorted(s["new_off"], t, right=True) - 1
    return seq, s["kv_len"][seq] - s["new_off"][seq + 1] + t


def _rotate(x, table, positions, rot, interleaved):
    half = rot // 2
    cos, sin = table[positions][:, None, :half], table[positions][:, None, half:]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:rot]
        y[..., :half], y[..., half:rot] = a * cos - b * sin, b * cos + a * sin
    return y


def _normed(x, w):
    if w is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()


def _begun(s):
    """The block that a sequence's first new token finds begun: page, first slot, tokens in it."""
    c = s["case"]
    first = s["kv_len"].long() - s["new_off"].diff()
    page = s["page_table"][torch.minimum(s["page_off"][:-1] + first // c["page"],
                                         s["page_off"][1:] - 1)].long()
    return page, first % c["page"] // c["block"] * c["block"], first % c["block"]


def _plain_append(s):
    c = s["case"]
    P, B = c["page"], c["block"]
    seq, pos = _rows(s)
    page = s["page_table"][s["page_off"][seq] + pos // P].long()
    slot = pos % P
    q = _rotate(_normed(s["q"].float(), s["q_norm"]), s["table"], pos, c["rot"], c["interleaved"])
    k = _rotate(_normed(s["k"].float(), s["k_norm"]), s["table"], pos, c["rot"], c["interleaved"])
    _plain_store(s["Kc"], s["Ks"], k, page, slot, _begun(s), B)
    _plain_store(s["Vc"], s["Vs"], s["v"].float(), page, slot, _begun(s), B)
    return q.to(s["q"].dtype)


def _plain_store(codes, scales, x, page, slot, begun, B):
    """New rows x [tokens, heads, dim] into their slots; scales of the blocks follow."""
    blocks = scales.shape[2]
    at = page * blocks + slot // B
    amax = torch.zeros(scales.shape[0] * blocks, scales.shape[1], device=DEV)
    amax.scatter_reduce_(0, at[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
    e = _exponent(amax).unflatten(0, (-1, blocks))                     # [pages, blocks, heads]
    # blocks that hold earlier tokens: the scale may only grow, and their codes follow it
    b_page, b_slot, b_have = begun
    old = scales[b_page, :, b_slot // B].int() - 127                   # [sequences, heads]
    have = b_have > 0
    e[b_page, b_slot // B] = torch.where(have[:, None], torch.maximum(e[b_page, b_slot // B], old),
                                         e[b_page, b_slot // B])
    grown = _power(old - e[b_page, b_slot // B])
    row = torch.arange(B, device=DEV)
    seq_i, row_i = (row < b_have[:, None]).nonzero(as_tuple=True)
    p_i, s_i = b_page[seq_i], b_slot[seq_i] + row_i
    codes[p_i, s_i] = (codes[p_i, s_i].float() * grown[seq_i, :, None]).to(codes.dtype)
    scales[page, :, slot // B] = (e[page, slot // B] + 127).to(torch.uint8)
    codes[page, slot] = (x * _power(-e[page, slot // B])[..., None]).to(codes.dtype)


def _gathered(s, name, seqs, width):
    """Keys or values of positions 0 .. width of the given sequences, padded, in 32 bits."""
    P, B = s["case"]["page"], s["case"]["block"]
    j = torch.arange(width, device=DEV).expand(len(seqs), -1)
    last = s["page_off"][seqs + 1] - 1
    at = torch.minimum(s["page_off"][seqs][:, None] + j // P, last[:, None])
    page = s["page_table"][at].long()
    scale = _power(s[name + "s"][page, :, j % P // B].int() - 127)
    return s[name + "c"][page, j % P].float().mul_(scale[..., None]), j


def _plain_attend(s):
    c = s["case"]
    every = torch.arange(c["n_seq"], device=DEV)
    t = s["new_off"][:-1, None] + torch.arange(s["max_new"], device=DEV)
    real = t < s["new_off"][1:, None]
    q = s["q"][t.clamp_max(s["n_new"] - 1)].float().unflatten(2, (c["hkv"], c["hq"] // c["hkv"]))
    k, j = _gathered(s, "K", every, s["max_kv"])
    pos = (s["kv_len"] - s["new_off"].diff())[:, None] + torch.arange(s["max_new"], device=DEV)
    x = torch.einsum("nthgd,njhd->nhgtj", q, k).mul_(s["scale"])
    x.masked_fill_(~(j[:, None] <= pos[..., None])[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min_(-1e30)
    p = x.sub_(m).exp_()
    del k
    v, _ = _gathered(s, "V", every, s["max_kv"])
    o = torch.einsum("nhgtj,njhd->nhgtd", p, v) / p.sum(-1, keepdim=True).clamp_min(1e-30)
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[real].to(s["q"].dtype)


def _plain_fork(s):
    """Counters of the old generation down, of the new one up; the lowest free pages, in the
    children's order, for the tokens behind the last whole page, which are copied."""
    c = s["case"]
    P, refs = c["page"], s["refs"]
    one = torch.ones((), dtype=torch.int32, device=DEV)
    refs.index_put_((s["kid_table"].long(),), -one, accumulate=True)
    pages = s["kid_off"].diff()
    kid = torch.repeat_interleave(torch.arange(len(pages), device=DEV), pages)
    local = torch.arange(len(s["kid_table"]), device=DEV) - s["kid_off"][kid]
    s["kid_table"].copy_(s["page_table"][s["page_off"][s["parent"].long()][kid] + local])
    tail = s["kid_len"] % P
    need = (tail > 0).nonzero().squeeze(1)
    fresh = (refs == 0).nonzero().squeeze(1)[:len(need)]
    last = s["kid_off"][need + 1] - 1
    source = s["kid_table"][last].long()
    s["kid_table"][last] = fresh.to(torch.int32)
    refs.index_put_((s["kid_table"].long(),), one, accumulate=True)
    body, page = _row_bytes(c)
    unit = 1 if c["block"] else 2
    row = body // P // unit
    i, r = (torch.arange(P, device=DEV) < tail[need, None]).nonzero(as_tuple=True)
    rows = s["pool_data"][..., :body // unit].unflatten(2, (P, row))
    rows[:, fresh[i], r] = rows[:, source[i], r]
    if page > body:
        scales = s["pool_data"][..., body:]
        scales[:, fresh] = scales[:, source]


def _plain_compact(s):
    """The k-th used page behind the first n goes to the k-th free one of the first n."""
    refs = s["refs"]
    used = refs > 0
    n = int(used.sum())
    source = used[n:].nonzero().squeeze(1) + n
    to = (~used[:n]).nonzero().squeeze(1)
    s["pool_data"][:, to] = s["pool_data"][:, source]
    place = torch.arange(len(refs), device=DEV)
    place[source] = to
    s["table_out"].copy_(place[s["page_table"].long()])
    s["refs_out"].copy_(refs)
    s["refs_out"][to] = refs[source]
    s["refs_out"][source] = 0
    s["n_live"].fill_(n)


# ---- the definition in 64 bits -----------------------------------------------------------

def exact(case, seed):
    """Sequence by sequence from the definitions, in 64 bits. Codes of new tokens are the values
    that they stand for in units of their block's scale, before the rounding to eight bits; the
    scales are powers of two chosen in 32 bits and have no further digits, nor have page calls."""
    if case["op"] in ("fork", "compact"):
        return None
    s = prepare(case, seed)
    new, kv = _shape(case)
    P, B, hq, hkv, d = (case[k] for k in ("page", "block", "hq", "hkv", "dim"))
    start, first_page = _cum(new), _cum([-(-b // P) for b in kv])
    if case["op"] == "append":
        rot = case["rot"]
        pos = torch.cat([torch.arange(b - a, b) for a, b in zip(new, kv)]).to(DEV)
        at = torch.cat([f + torch.arange(b - a, b) // P
                        for a, b, f in zip(new, kv, first_page)]).to(DEV)
        page = s["page_table"].long()[at]
        cos, sin = (x[:, None].double() for x in s["table"][pos].split(rot // 2, 1))
        done = []
        for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
            x = x.double()
            if w is not None:
                x = x / ((x * x).sum(-1, keepdim=True) / d + 1e-6).sqrt() * w.double()
            z, rest = x[..., :rot], x[..., rot:]
            z = z.unflatten(-1, (-1, 2)).transpose(-1, -2) if case["interleaved"] \
                else z.unflatten(-1, (2, -1))
            z = torch.stack([z[..., 0, :] * cos - z[..., 1, :] * sin,
                             z[..., 1, :] * cos + z[..., 0, :] * sin], -2)
            z = z.transpose(-1, -2) if case["interleaved"] else z
            done.append(torch.cat([z.flatten(-2), rest], -1))
        out = [done[0]]
        for name, x in (("K", done[1]), ("V", s["v"].double())):
            codes = s[name + "c"].double()
            scales = s[name + "s"].long().transpose(1, 2) - 127        # [pages, blocks, heads]
            # least exponent whose largest code reaches a row's largest element
            want = torch.ceil(torch.log2(x.abs().amax(-1) / 448)).clamp(E_MIN, E_MAX).long()
            e = torch.full(scales.shape, E_MIN, device=DEV)
            flat = (page * (P // B) + pos % P // B)[:, None].expand(-1, hkv)
            e.view(-1, hkv).scatter_reduce_(0, flat, want, "amax")
            for i, (a, b) in enumerate(zip(new, kv)):
                p0 = b - a
                if p0 % B:
                    pg, blk = int(s["page_table"][first_page[i] + p0 // P]), p0 % P // B
                    e[pg, blk] = torch.maximum(e[pg, blk], scales[pg, blk])
                    codes[pg, blk * B:p0 % P] *= torch.exp2((scales[pg, blk] - e[pg, blk]).double())[:, None]
            codes[page, pos % P] = x * torch.exp2(-e[page, pos % P // B].double())[..., None]
            out += [codes, None]
        return tuple(out)
    out = torch.empty(start[-1], hq, d, dtype=torch.float64, device=DEV)
    for i, (a, b) in enumerate(zip(new, kv)):
        pages = s["page_table"][first_page[i]:first_page[i + 1]].long()
        k, v = ((s[x + "c"][pages].double().unflatten(1, (-1, B)) *
                 torch.exp2(s[x + "s"][pages].double() - 127).transpose(1, 2)[:, :, None, :, None])
                .flatten(0, 2)[:b] for x in "KV")
        limit = torch.arange(b - a, b, device=DEV)[:, None]
        hidden = torch.arange(b, device=DEV)[None] > limit
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            q = s["q"][start[i]:start[i + 1], heads].double().transpose(0, 1)
            x = (q @ k[:, h].T) / math.sqrt(d)
            w = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[start[i]:start[i + 1], heads] = (w @ v[:, h]).transpose(0, 1)
    return out
