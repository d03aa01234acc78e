"""The 8-bit key/value cache in 64 bits, for the tests: its format, the append and the attention, from their definitions."""
import math

import torch

E4M3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()   # the non-negative values, by code
MIDDLE = (E4M3[1:] + E4M3[:-1]) / 2


def values(codes, scales):
    """Codes [.., d] and scale bytes [.., d / 32] (uint8) as the values they stand for."""
    x = codes.view(torch.float8_e4m3fn).double().unflatten(-1, (-1, 32))
    return (x * torch.exp2(scales.double() - 127)[..., None]).flatten(-2)


def mxfp8(y):
    """MXFP8 of y [.., d] (fp64): codes and scale bytes; e = floor(log2 amax) - 8 (never below -127), nearest even, saturating."""
    b = y.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1)
    e = torch.where(amax > 0, torch.floor(torch.log2(amax.clamp(min=1e-300))) - 8, torch.full_like(amax, -127.0)).clamp(min=-127)
    u = b / torch.exp2(e)[..., None]
    a = u.abs().contiguous()
    low, high = torch.searchsorted(MIDDLE, a), torch.searchsorted(MIDDLE, a, right=True)
    code = torch.where(low % 2 == 0, low, high).to(torch.uint8) | (torch.signbit(u).to(torch.uint8) << 7)
    return code.flatten(-2), (e + 127).to(torch.uint8)


def rotate(x, table_rows):
    """x [tokens, heads, d] fp64; table_rows [tokens, rot]: cosines, then sines."""
    r = table_rows.shape[1]
    cos, sin = table_rows.double()[:, None].chunk(2, -1)
    a, b, rest = x[..., :r // 2], x[..., r // 2:r], x[..., r:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def dense(left, right, k):
    """[k, 32, 32]: the block matrices L_j (x) R_j."""
    left, right = torch.as_tensor(left).double(), torch.as_tensor(right).double()
    return torch.stack([torch.kron(left[min(j, left.shape[0] - 1)], right[min(j, right.shape[0] - 1)]) for j in range(k)])


def transform(x, p):
    return torch.einsum("thkc,kcd->thkd", x.unflatten(-1, (-1, 32)), p).flatten(-2)


def clip(x, lo, hi):
    b = x.unflatten(-1, (-1, 32))
    lo, hi = torch.as_tensor(lo).double()[:, None], torch.as_tensor(hi).double()[:, None]
    return torch.minimum(torch.maximum(b, lo * b.amin(-1, keepdim=True)), hi * b.amax(-1, keepdim=True)).flatten(-2)


def gather(codes, scales, ids, n):
    """The first n tokens on the pages `ids`: [kv_heads, n, d] in fp64."""
    return values(codes[ids], scales[ids]).transpose(0, 1).flatten(1, 2)[:, :n]


def attention(q, k_cache, v_cache, rows, lens, pages, scale, causal, hidden=None):
    """q [tokens, heads, d] (any type, CPU); k_cache, v_cache: (codes, scales) on the CPU; pages: a list of page lists.
    Returns out, lse, and a bound on how far the kernel may be off before its last rounding:

      weights   each is off by 2^-11 of itself (f16) plus 2^-25 of the row's largest weight times 2^c of its tile of 32
                tokens, c the exponent that the tile's values are divided by;
      scores    fp32 sums of exact products, in any order: (d + 8) 2^-24 sum |q k| scale, and a few fp32 roundings of the
                score and of its exponential, 2^-20 in all, which count twice (numerator and denominator);
      sums      fp32, n 2^-24 relative each, numerator and denominator, and products exact.
    """
    heads, d = q.shape[1], q.shape[2]
    kv_heads = k_cache[0].shape[1]
    group = heads // kv_heads
    total = q.shape[0]
    out, lse, bound = torch.zeros(total, heads, d, dtype=torch.float64), torch.full((total, heads), -math.inf, dtype=torch.float64), torch.zeros(
        total, heads, d, dtype=torch.float64)
    at = 0
    for i, (m, n) in enumerate(zip(rows, lens)):
        if n > 0 and m > 0:
            k, v = gather(*k_cache, pages[i], n), gather(*v_cache, pages[i], n)
            gone = torch.zeros(n, dtype=torch.bool) if hidden is None else hidden[i][:n]
            k, v = k.masked_fill(gone[:, None], 0.0), v.masked_fill(gone[:, None], 0.0)
            c = v.abs().amax(dim=(0, 2))
            c = torch.nn.functional.pad(c, (0, -n % 32)).unflatten(0, (-1, 32)).amax(1).clamp(min=1e-30)
            c = torch.exp2(torch.floor(torch.log2(c))).repeat_interleave(32)[:n]    # 2^c up to a common factor of 2^15
            qs = q[at:at + m].double().transpose(0, 1).unflatten(0, (kv_heads, group))       # [hk, group, m, d]
            s = torch.einsum("hgmd,hnd->hgmn", qs, k) * scale
            see = torch.arange(n) <= (torch.arange(m)[:, None] + n - m if causal else torch.full((m, 1), n))
            see = see & ~gone
            s = s.masked_fill(~see, -math.inf)
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
            l = w.sum(-1, keepdim=True)
            p = w / l.clamp(min=1e-300)
            o = torch.einsum("hgmn,hnd->hgmd", p, v)
            off = torch.einsum("hgmd,hnd->hgmn", qs.abs(), k.abs()) * abs(scale) * (d + 8) * 2.0 ** -24 + 2.0 ** -20
            off = off.masked_fill(~see, 0.0)
            a = torch.einsum("hgmn,hnd->hgmd", p, v.abs())
            rel = 2.0 ** -11 + off + n * 2.0 ** -24
            b = torch.einsum("hgmn,hnd->hgmd", p * rel, v.abs()) + a * ((p * off).sum(-1, keepdim=True) + n * 2.0 ** -24)
            # 2^-25 of the largest weight: p 2^c over the row, met by values of |v| / 2^c <= 2 (in the same units)
            big = (p * c).amax(-1, keepdim=True)
            b = b + 2.0 ** -25 * big * torch.einsum("hgmn,hnd->hgmd", see.double().expand_as(p), v.abs() / c[:, None])
            out[at:at + m] = o.flatten(0, 1).transpose(0, 1)
            bound[at:at + m] = b.flatten(0, 1).transpose(0, 1)
            x = torch.where(l > 0, top + torch.log(l.clamp(min=1e-300)), torch.full_like(l, -math.inf))
            lse[at:at + m] = x.squeeze(-1).flatten(0, 1).transpose(0, 1)
        at += m
    return out, lse, bound
