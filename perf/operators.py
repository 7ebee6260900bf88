"""Cases of the operators around the paged pool: append (norm + rotation + write), attend and
attend over shared prefixes.

Sizes follow this repository's workloads: the Llama-3-8B KV shape (8 KV heads of 128, pages of 16,
256 requests of 1k to 8k tokens with Zipf-shared prefixes of 512 to 4k), the small-head GQA shape
(4 KV heads, pages of 64, 512 conversations, turns of 256 to 1024 tokens) and the long-context shape
(8 KV heads under 64 query heads, requests of 32768 tokens whose last 1k changed).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_contexts = {}


# ---- cases -------------------------------------------------------------------------------

def _case(name, op, dtype, hq, hkv, dim, page, n_seq, new, hist, shape_seed=1, norm=False,
          rot=0, interleaved=False, groups=0, shared=(0, 0)):
    c = {"op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "dim": dim, "page": page,
         "n_seq": n_seq, "new_lo": new[0], "new_hi": new[1], "hist_lo": hist[0],
         "hist_hi": hist[1], "shape_seed": shape_seed}
    if op == "append":
        c.update(norm=norm, rot=rot or dim, interleaved=interleaved)
    if op == "shared":
        c.update(groups=groups, shared_lo=shared[0], shared_hi=shared[1])
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step of a lightly loaded server: latency counts
        _case("append_step_8", "append", "bf16", 32, 8, 128, 16, 8, (1, 1), (100, 1000)),
        # a full decode step of a model that normalises queries and keys per head
        _case("append_step_512_norm", "append", "bf16", 28, 4, 128, 64, 512, (1, 1), (64, 1024),
              norm=True),
        # the next turn of 64 conversations enters the cache
        _case("append_turn", "append", "fp16", 28, 4, 128, 64, 64, (256, 1024), (0, 2048),
              norm=True),
        # a decode step of four short chats: latency counts
        _case("attend_step_4", "attend", "bf16", 32, 8, 128, 16, 4, (1, 1), (200, 1000)),
        # a decode step of the Llama-3-8B-shaped workload, every request with its own cache
        _case("attend_step_llama8b", "attend", "bf16", 32, 8, 128, 16, 256, (1, 1), (1023, 8191)),
        # a decode step of 512 conversations on four KV heads
        _case("attend_step_gqa4", "attend", "fp16", 28, 4, 128, 64, 512, (1, 1), (256, 4096)),
        # what is left of 32 prompts after their stored prefixes were restored, from one token on
        _case("attend_suffix", "attend", "bf16", 32, 8, 128, 16, 32, (1, 512), (512, 4096)),
        # two long-context requests whose last 1k tokens changed
        _case("attend_long", "attend", "bf16", 64, 8, 128, 16, 2, (1024, 1024), (31744, 31744)),
        # fresh prompts of a model with as many KV heads as query heads, heads of 64
        _case("attend_prefill_64", "attend", "fp16", 16, 16, 64, 16, 6, (700, 3000), (0, 0)),
        # eight samples of one prompt a few tokens in: latency counts
        _case("shared_step_8", "shared", "bf16", 32, 8, 128, 16, 8, (1, 1), (0, 63), groups=1,
              shared=(1024, 1024)),
        # a decode step of the Llama-3-8B-shaped workload with its 64 shared prefixes
        _case("shared_step_llama8b", "shared", "bf16", 32, 8, 128, 16, 256, (1, 1), (511, 4095),
              groups=64, shared=(512, 4096)),
        # 64 requests over one long document
        _case("shared_step_long", "shared", "fp16", 64, 8, 128, 16, 64, (1, 1), (63, 1023),
              groups=1, shared=(16384, 16384)),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng: random.Random):
    op = rng.choice(("append", "attend", "attend", "shared"))
    hq, hkv = rng.choice(((32, 8), (28, 4), (64, 8), (16, 16), (24, 4), (16, 2), (40, 8)))
    dim = rng.choice((64, 96, 128, 128))
    page = rng.choice((16, 16, 32, 64))
    dtype = rng.choice(("bf16", "fp16"))
    seed = rng.randrange(1, 1 << 30)
    if op == "append":
        n_seq = _log(rng, 1, 512)
        hi = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, min(4096, 40000 // n_seq)))
        return _case(None, op, dtype, hq, hkv, dim, page, n_seq, (1, hi), (0, _log(rng, 8, 1024)),
                     seed, norm=rng.random() < 0.5, rot=rng.choice((dim, dim, dim // 2)),
                     interleaved=rng.random() < 0.3)
    if op == "attend":
        if rng.random() < 0.5:                                        # one token each
            n_seq = _log(rng, 1, 512)
            hi = _log(rng, 16, max(16, min(65536, 1000000 // n_seq)))
            return _case(None, op, dtype, hq, hkv, dim, page, n_seq, (1, 1), (hi // 5, hi), seed)
        n_seq = _log(rng, 1, 32)                                      # a suffix or a prompt
        new = _log(rng, 2, 2048)
        hist = _log(rng, 1, 16384)
        while n_seq > 1 and n_seq * hq * new * (new + hist) > 4e9:
            n_seq //= 2
        while n_seq * hq * new * (new + hist) > 4e9:
            new = (new + 1) // 2
        return _case(None, op, dtype, hq, hkv, dim, page, n_seq, (1, new), (hist // 3, hist), seed)
    groups = _log(rng, 1, 32)
    n_seq = groups * _log(rng, 2, max(2, 256 // groups))
    shared = _log(rng, 100, max(100, min(16384, 200000 // groups)))
    hist = _log(rng, 1, max(1, min(2048, 400000 // n_seq)))
    return _case(None, op, dtype, hq, hkv, dim, page, n_seq, (1, 1), (hist // 4, hist), seed,
                 groups=groups, shared=(shared // 2, shared))


# ---- lengths and page tables -------------------------------------------------------------

def _shape(case):
    """new, kv, group of every sequence and the shared length of every group: the case's own."""
    r = random.Random(case["shape_seed"])
    n = case["n_seq"]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    kv = [a + r.randint(case["hist_lo"], case["hist_hi"]) for a in new]
    group_off, shared = None, None
    if case["op"] == "shared":
        g = case["groups"]
        # whole pages, as the store restores them
        shared = [max(1, r.randint(case["shared_lo"], case["shared_hi"]) // case["page"])
                  * case["page"] for _ in range(g)]
        # every group has a sequence; the others fall on the groups by Zipf's law
        size = [1] * g
        weight = [1.0 / (k + 1) ** 1.1 for k in range(g)]
        for k in r.choices(range(g), weight, k=n - g):
            size[k] += 1
        group_off = [0]
        for k in range(g):
            for i in range(group_off[-1], group_off[-1] + size[k]):
                kv[i] += shared[k]
            group_off.append(group_off[-1] + size[k])
    return new, kv, group_off, shared


def _cum(v):
    out = [0]
    for x in v:
        out.append(out[-1] + x)
    return out


def work(case):
    new, kv, group_off, shared = _shape(case)
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    row = d * 2
    t = sum(new)
    if case["op"] == "append":
        heads = hq + 2 * hkv
        table = t * case["rot"] * 4
        pairs = t * (hq + hkv) * case["rot"] / 2
        norm = 4 * t * (hq + hkv) * d if case["norm"] else 0
        return {"bytes": 2 * t * heads * row + table + 4 * t, "flops": 6 * pairs + norm}
    seen = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(new, kv))
    read = sum(kv)
    if case["op"] == "shared":
        for k, s in enumerate(shared):
            members = group_off[k + 1] - group_off[k]
            read -= (members - 1) * s
    return {"bytes": 2 * read * hkv * row + 2 * t * hq * row + 4 * (read // case["page"]),
            "flops": 4 * seen * hq * d}


def prepare(case, seed):
    new, kv, group_off, shared = _shape(case)
    dt = DTYPES[case["dtype"]]
    P, hq, hkv, d = case["page"], case["hq"], case["hkv"], case["dim"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + case["shape_seed"])

    def normal(*shape, scale=1.0):
        x = torch.randn(shape, generator=g, device=DEV, dtype=dt)
        return x if scale == 1.0 else x.mul_(scale)

    # a fragmented pool: pages in random order, a group's shared whole pages in common
    pages = [-(-b // P) for b in kv]
    common = [0] * len(kv)
    if group_off is not None:
        for k, s in enumerate(shared):
            for i in range(group_off[k] + 1, group_off[k + 1]):
                common[i] = s // P
    fresh = _cum([a - b for a, b in zip(pages, common)])
    page_off = _cum(pages)
    num_pages = fresh[-1] + 8
    perm = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32)
    slot = torch.arange(page_off[-1], dtype=torch.int64)
    owner = torch.repeat_interleave(torch.arange(len(kv)), torch.tensor(pages))
    local = slot - torch.tensor(page_off)[owner]
    take = torch.tensor(fresh)[owner] + local - torch.tensor(common)[owner]
    if group_off is not None:
        first = torch.repeat_interleave(torch.tensor(group_off[:-1]),
                                        torch.tensor(group_off).diff())[owner]
        take = torch.where(local < torch.tensor(common)[owner], torch.tensor(fresh)[first] + local,
                           take)
    s = {
        "case": dict(case), "op": case["op"], "scale": d ** -0.5,
        "n_new": sum(new), "max_new": max(new), "max_kv": max(kv),
        "new_off": torch.tensor(_cum(new), device=DEV),
        "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
        "page_off": torch.tensor(page_off, device=DEV),
        "page_table": perm[take.to(DEV)].contiguous(),
        "K": normal(num_pages, P, hkv, d), "V": normal(num_pages, P, hkv, d),
    }
    s["pool"] = (torch.tensor([s["K"].data_ptr(), s["V"].data_ptr()], device=DEV), num_pages)
    if case["op"] == "append":
        # what the projection of a layer leaves: q, k and v of a token side by side
        qkv = normal(sum(new), hq + 2 * hkv, d)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
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
    if case["op"] == "shared":
        s["group_off"] = torch.tensor(group_off, dtype=torch.int32, device=DEV)
        s["shared_pages"] = torch.tensor(shared, dtype=torch.int32, device=DEV) // P
        s["max_shared"], s["max_own"] = max(shared), max(
            kv[i] - shared[k] for k in range(len(shared))
            for i in range(group_off[k], group_off[k + 1]))
        s["max_member"] = max(b - a for a, b in zip(group_off, group_off[1:]))
    if own:
        # the handle and the step's descriptors, which a serving loop keeps over all its layers
        from paper_2511_16138_b200 import lsmkv
        geom = lsmkv.Geom(n_layers=1, n_kv_heads=hkv, head_dim=d, page_tokens=P, chunk_tokens=P)
        if geom not in _contexts:
            _contexts[geom] = lsmkv.Context(geom, torch.cuda.current_device())
        s["ctx"] = _contexts[geom]
        s["seqs"] = lsmkv.Seqs(s["new_off"], s["kv_len"], s["page_off"], s["page_table"],
                               s["n_new"], s["max_new"])
        if case["op"] == "append":
            s["rope"] = lsmkv.Rope(s["table"], interleaved=case["interleaved"])
        if case["op"] == "shared":
            s["groups"] = lsmkv.Groups(s["group_off"], s["shared_pages"])
    return s


# ---- the operators -----------------------------------------------------------------------

def run(s):
    if own:
        if s["op"] == "append":
            s["ctx"].append_batch(0, s["seqs"], s["k"], s["v"], s["pool"], rope=s["rope"],
                                  q=s["q"], q_out=s["out"], q_norm=s["q_norm"],
                                  k_norm=s["k_norm"], eps=1e-6)
            return s["out"], s["K"], s["V"]
        if s["op"] == "attend":
            s["ctx"].attend_batch(0, s["seqs"], s["q"], s["out"], s["pool"], s["scale"])
        else:
            s["ctx"].attend_shared_batch(0, s["seqs"], s["groups"], s["q"], s["out"], s["pool"],
                                         s["scale"])
        return s["out"]
    if s["op"] == "append":
        return _plain_append(s)
    return _plain_attend(s) if s["op"] == "attend" else _plain_shared(s)


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


def _plain_append(s):
    c = s["case"]
    seq, pos = _rows(s)
    page = s["page_table"][s["page_off"][seq] + pos // c["page"]].long()
    slot = pos % c["page"]
    q = _rotate(_normed(s["q"].float(), s["q_norm"]), s["table"], pos, c["rot"], c["interleaved"])
    k = _rotate(_normed(s["k"].float(), s["k_norm"]), s["table"], pos, c["rot"], c["interleaved"])
    s["K"][page, slot] = k.to(s["K"].dtype)
    s["V"][page, slot] = s["v"]
    return q.to(s["K"].dtype), s["K"], s["V"]


def _gathered(s, first, seqs, start, width):
    """K and V of positions start .. start + width of the given sequences, padded, in 32 bits."""
    P = s["case"]["page"]
    j = start[:, None] + torch.arange(width, device=DEV)
    last = s["page_off"][seqs + 1] - 1
    at = torch.minimum(s["page_off"][first][:, None] + j // P, last[:, None])
    page = s["page_table"][at].long()
    return s["K"][page, j % P].float(), s["V"][page, j % P].float(), j


def _parts(q, k, v, seen, scale):
    """Maximum, sum and weighted sum of the visible keys: q [n, t, hkv, g, d], seen [n, t, j]."""
    x = torch.einsum("nthgd,njhd->nhgtj", q, k).mul_(scale)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min_(-1e30)
    p = x.sub_(m).exp_()
    return m, p.sum(-1, keepdim=True), torch.einsum("nhgtj,njhd->nhgtd", p, v)


def _padded(s, off, width):
    """The queries of a run of tokens per row of `off`, padded to `width` tokens."""
    c = s["case"]
    t = off[:-1, None] + torch.arange(width, device=DEV)
    q = s["q"][t.clamp_max(s["n_new"] - 1)].float()
    return q.unflatten(2, (c["hkv"], c["hq"] // c["hkv"])), t < off[1:, None]


def _flat(o, real):
    """[n, hkv, g, t, d] -> the real tokens, [tokens, hq, d]"""
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[real]


def _plain_attend(s):
    n = s["case"]["n_seq"]
    every = torch.arange(n, device=DEV)
    q, real = _padded(s, s["new_off"], s["max_new"])
    k, v, j = _gathered(s, every, every, torch.zeros_like(every), s["max_kv"])
    new = s["new_off"].diff()
    pos = (s["kv_len"] - new)[:, None] + torch.arange(s["max_new"], device=DEV)
    m, l, o = _parts(q, k, v, j[:, None] <= pos[..., None], s["scale"])
    return _flat(o / l.clamp_min(1e-30), real).to(s["q"].dtype)


def _plain_shared(s):
    n = s["case"]["n_seq"]
    every = torch.arange(n, device=DEV)
    sizes = s["group_off"].diff()
    group = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), sizes)
    first = s["group_off"][:-1].long()
    # the shared part, once for the tokens of a group
    off = s["new_off"][s["group_off"].long()]
    width = s["max_member"] * s["max_new"]
    q, real = _padded(s, off, width)
    k, v, j = _gathered(s, first, first, torch.zeros_like(first), s["max_shared"])
    shared = s["shared_pages"].long() * s["case"]["page"]
    seen = (j < shared[:, None])[:, None].expand(-1, width, -1)
    m1, l1, o1 = (_flat(x, real) for x in _parts(q, k, v, seen, s["scale"]))
    # every sequence's own part
    q, real = _padded(s, s["new_off"], s["max_new"])
    start = shared[group]
    k, v, j = _gathered(s, every, every, start, s["max_own"])
    new = s["new_off"].diff()
    pos = (s["kv_len"] - new)[:, None] + torch.arange(s["max_new"], device=DEV)
    m2, l2, o2 = (_flat(x, real) for x in _parts(q, k, v, j[:, None] <= pos[..., None],
                                                 s["scale"]))
    m = torch.maximum(m1, m2)
    a, b = (m1 - m).exp(), (m2 - m).exp()
    return ((a * o1 + b * o2) / (a * l1 + b * l2)).to(s["q"].dtype)


# ---- the definition in 64 bits -----------------------------------------------------------

def exact(case, seed):
    """Sequence by sequence from the definitions, in 64 bits."""
    s = prepare(case, seed)
    new, kv, _, _ = _shape(case)
    P, hq, hkv, d = case["page"], case["hq"], case["hkv"], case["dim"]
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
        K, V = s["K"].double(), s["V"].double()
        K[page, pos % P] = done[1]
        V[page, pos % P] = s["v"].double()
        return done[0], K, V
    out = torch.empty(start[-1], hq, d, dtype=torch.float64, device=DEV)
    for i, (a, b) in enumerate(zip(new, kv)):
        pages = s["page_table"][first_page[i]:first_page[i + 1]].long()
        k, v = (x[pages].flatten(0, 1)[:b].double() for x in (s["K"], s["V"]))
        limit = torch.arange(b - a, b, device=DEV)[:, None]
        hidden = torch.arange(b, device=DEV)[None] > limit
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            q = s["q"][start[i]:start[i + 1], heads].double().transpose(0, 1)
            x = (q @ k[:, h].T) / math.sqrt(d)
            w = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[start[i]:start[i + 1], heads] = (w @ v[:, h]).transpose(0, 1)
    return out
