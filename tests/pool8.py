"""Helpers of the tests on 8-bit pools: buffers, their views, and the values that they stand for."""
import torch

from paper_2511_16138_b200 import lsmkv

DEV = "cuda:0"


def geom8(n_layers, hkv, D, P, B):
    return lsmkv.Geom(n_layers, hkv, D, elem_bytes=1, page_tokens=P, chunk_tokens=P,
                      flags=lsmkv.pool_e4m3(B))


def views(pool, g):
    """Codes [2L, pages, P, hkv, D] and scale bytes [2L, pages, hkv, P / B] of a pool [2L, pages, page_bytes]."""
    P, H, D, B = g.page_tokens, g.n_kv_heads, g.head_dim, g.block_tokens
    codes = pool[..., :g.code_bytes].view(torch.float8_e4m3fn).unflatten(-1, (P, H, D))
    scales = pool[..., g.code_bytes:g.code_bytes + H * (P // B)].unflatten(-1, (H, P // B))
    return codes, scales


def exponents(scales):
    return (scales.long() - 127).clamp(-100, 100)


def values(pool, g, dtype=torch.float64):
    """What the codes stand for, [2L, pages, P, hkv, D]."""
    codes, scales = views(pool, g)
    e = exponents(scales).transpose(-1, -2)                              # [2L, pages, blocks, hkv]
    x = codes.to(dtype).unflatten(2, (-1, g.block_tokens))
    return (x * torch.exp2(e.to(dtype))[:, :, :, None, :, None]).flatten(2, 3)


def least_exponent(amax):
    """ceil(log2(amax / 448)) within -100..100, for amax in 64 bits."""
    m, e = torch.frexp(amax.clamp_min(1e-300) / 448)                      # m in [0.5, 1)
    return torch.where(m == 0.5, e - 1, e).long().clamp(-100, 100)


def filled(g, num, generator, spread=None):
    """A pool whose pages hold normal values, every block with its least exponent."""
    pool = torch.zeros(2 * g.n_layers, num, g.page_bytes, dtype=torch.uint8, device=DEV)
    codes, scales = views(pool, g)
    x = torch.randn(codes.shape, generator=generator, device=DEV)
    if spread is not None:
        x = x * spread
    x = x.unflatten(2, (-1, g.block_tokens))
    e = least_exponent(x.abs().amax((3, 5)).double())                     # [2L, pages, blocks, hkv]
    codes.copy_((x * torch.exp2(-e.float())[:, :, :, None, :, None]).flatten(2, 3).to(codes.dtype))
    scales.copy_((e + 127).transpose(-1, -2).to(torch.uint8))
    return pool
