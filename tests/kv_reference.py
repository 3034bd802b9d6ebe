"""The paged cache and the attention over it in 64 bits on the CPU, element by element from the layout and the formulas that
include/skd.h gives."""
import math

import numpy as np
import torch

BF16, FP8 = 0, 1


def round_e4m3(y):
    """float64 magnitudes up to 448 rounded to e4m3 (4 significant bits, multiples of 2^-9 below 2^-6), halves to even."""
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.round(y / step) * step


def e4m3_values():
    """The value of each code 0 .. 255."""
    c = np.arange(256)
    e, m, s = c >> 3 & 15, c & 7, np.where(c > 127, -1.0, 1.0)
    v = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * np.exp2(e - 7.0))
    return np.where((c & 127) == 127, np.nan, s * v)


def exponent(x):
    """Exponent byte of each vector along the last axis."""
    a = np.abs(x).max(-1)
    with np.errstate(all="ignore"):
        e = np.ceil(np.log2(a / 448.0))
        e = np.where(a > 448.0 * np.exp2(e), e + 1, np.where(a <= 224.0 * np.exp2(e), e - 1, e))
    e = np.where(np.isfinite(e), np.maximum(e, -127), -127)
    return np.where(np.isfinite(a), e + 127, 255).astype(np.int64)


def as_held(x, elem):
    """What a page holds of x [..., dh] (float64 of bf16 values), as values."""
    if elem == BF16:
        return x
    b = exponent(x)
    with np.errstate(all="ignore"):
        s = np.exp2(b - 127.0)[..., None]
        y = round_e4m3(x / s)
        y = np.where((b == 247)[..., None], np.clip(y, -240.0, 240.0), y) * s
    return np.where((b == 255)[..., None], np.nan, y)


def unpack_page(page, elem, H, dh, page_tokens):
    """K, V [page_tokens][H][dh] float64 of one page given as int16 (bf16 bits) or uint8."""
    K, V = np.zeros((page_tokens, H, dh)), np.zeros((page_tokens, H, dh))
    p, e = np.arange(page_tokens)[:, None], np.arange(dh)[None, :]
    s, x, pos = p % 32, p % 32 // 16, p % 16
    for h in range(H):
        block = (h * (page_tokens // 32) + p // 32) * 64 * dh
        if elem == BF16:
            k = block + ((x * (dh // 32) + e // 32) * 4 + e % 32 // 8) * 128 + pos * 8 + e % 8
            v = block + 32 * dh + ((e // 16 * 4 + pos // 4) * 16 + e % 16) * 8 + x * 4 + pos % 4
            bits = page.astype(np.int64) & 0xffff
            for dst, at in ((K, k), (V, v)):
                dst[:, h] = (bits[at].astype(np.uint32) << 16).view(np.float32)
        else:
            k = block + ((x * (dh // 64) + e // 64) * 4 + e % 32 // 8) * 256 + pos * 16 + e // 32 % 2 * 8 + e % 8
            v = block + 32 * dh + ((e // 32 * 4 + pos // 4) * 16 + e % 16) * 16 + e // 16 % 2 * 8 + x * 4 + pos % 4
            exps = H * page_tokens * 2 * dh + (h * (page_tokens // 32) + p // 32) * 64 + s
            values = e4m3_values()
            for dst, at, ex in ((K, k, exps), (V, v, exps + 32)):
                b = page[ex].astype(np.int64)
                dst[:, h] = np.where(b == 255, np.nan, values[page[at]] * np.exp2(b - 127.0))
    return K, V


def attention(q, k, v, past, scale):
    """One row: q [new][heads][dh], k, v [past + new][kv heads][dh] float64.  Returns (out, bound): what a kernel may be off that
    rounds weights and output to bf16, in fp32 otherwise.

    Weights are rounded by at most 2^-8 of themselves, in numerator and denominator alike, so an output moves by at most 2^-8 *
    sum_j w_j |v_j - o| (w: the softmax); the output by 2^-8 of itself.  A score is a sum of dh products in fp32 and a product:
    off by (dh + 4) * 2^-24 of scale * sum |q||k|, and the weight by that fraction, the exponential's argument by 2^-23 of the
    difference of two scores, the exponential by 2^-22, sums over the keys by a multiple of 2^-24 that grows with their number's
    logarithm at least and is covered by 2^-18."""
    new, heads, dh = q.shape
    group = heads // k.shape[1]
    out, bound = torch.zeros(new, heads, dh, dtype=torch.float64), torch.zeros(new, heads, dh, dtype=torch.float64)
    for h in range(heads):
        kh, vh = k[:, h // group], v[:, h // group]
        s = q[:, h] @ kh.t() * scale
        size = (q[:, h].abs() @ kh.abs().t() * scale)
        seen = torch.arange(kh.shape[0])[None] <= past + torch.arange(new)[:, None]
        s = torch.where(seen, s, -math.inf)
        w = torch.softmax(s, -1)
        finite = torch.where(seen[..., None], vh[None], 0.0) if not torch.isfinite(vh).all() else None
        o = w @ vh if finite is None else (w[..., None] * finite).sum(1)
        big = torch.where(seen, size, 0.0).amax(-1, keepdim=True)
        eps = 2.0 ** -8 * 1.01 + (dh + 4) * 2.0 ** -23 * big + 2.0 ** -18
        spread = (w[..., None] * ((vh[None] if finite is None else finite) - o[:, None]).abs()).sum(1)
        out[:, h] = o
        bound[:, h] = eps * spread + 2.0 ** -8 * 1.01 * o.abs() + 2.0 ** -18 * (w @ vh.abs() if finite is None else spread + o.abs()) + 1e-37
    return out, bound
