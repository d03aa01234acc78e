"""Attention where one token has nearly all of the probability and next to no values (the first token of many models): what
the others add is the output, and their weights are small against the largest one."""
import math

import pytest
import torch

import kv_reference as R
from test_gpu_kv_cache import Append

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[1, 2], ids=["codes", "copy"])
def copy_path(batq, request):
    batq.batq_debug_force_attention_copy(request.param)
    yield request.param
    batq.batq_debug_force_attention_copy(0)


def _reference(q, k, v, scale):
    """One sequence, causal from its end.  q [m, heads, d], k, v [kv_heads, n, d] in 64 bits: out [m, heads, d] and how far
    the kernels may be off before the last rounding.  With e_t the power of two at or below the largest of token t's values
    (2^-49 at least) and C the row's largest p_t e_t:
      weights   2^-11 of themselves (f16), plus 2^-24 C / e_t each;
      scores    (d + 8) 2^-24 sum |q k| scale and 2^-20, twice (numerator and denominator);
      sums      n 2^-24, numerator and denominator."""
    m, heads, d = q.shape
    n, group = k.shape[1], heads // k.shape[0]
    qs = q.double().transpose(0, 1).unflatten(0, (-1, group))
    see = torch.arange(n) <= torch.arange(m)[:, None] + n - m
    p = torch.softmax((torch.einsum("hgmd,hnd->hgmn", qs, k) * scale).masked_fill(~see, -math.inf), -1)
    off = torch.einsum("hgmd,hnd->hgmn", qs.abs(), k.abs()) * scale * (d + 8) * 2.0 ** -24 + 2.0 ** -20
    e = torch.exp2(torch.floor(torch.log2(v.abs().amax(-1).clamp(min=2.0 ** -49))))        # [hk, n]
    out = torch.einsum("hgmn,hnd->hgmd", p, v)
    bound = torch.einsum("hgmn,hnd->hgmd", p * (2.0 ** -11 + off + n * 2.0 ** -24), v.abs())
    bound += torch.einsum("hgmn,hnd->hgmd", p, v.abs()) * ((p * off).sum(-1, keepdim=True) + n * 2.0 ** -24)
    most = (p * e[:, None, None]).amax(-1, keepdim=True)
    bound += 2.0 ** -24 * most * torch.einsum("hgmn,hnd->hgmd", see.double().expand_as(p), v.abs() / e[..., None])
    return out.flatten(0, 1).transpose(0, 1), bound.flatten(0, 1).transpose(0, 1)


def _attend(batq, q, k, v, page):
    """q [m, heads, d] bf16; k, v [n, kv_heads, d]: through a cache whose pages stand in order.  Output and keys, values as the codes are."""
    n, kv_heads, d = k.shape
    pages = n // page
    stored = [R.mxfp8(x.double().unflatten(0, (pages, page)).transpose(1, 2).contiguous()) for x in (k, v)]
    cache = batq.batq_kv_cache_create(*[y.cuda() for x in stored for y in x])
    m, heads = q.shape[:2]
    out = torch.full((m, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(cache, heads, m, 1, m, n))
    batq.batq_attention_kv_mxfp8(cache, q.cuda().flatten(1), out, torch.tensor([n], dtype=torch.int32, device="cuda"),
                                 torch.arange(pages, dtype=torch.int32, device="cuda")[None], m, n, ws,
                                 q_starts=torch.tensor([0, m], dtype=torch.int32, device="cuda"))
    assert batq.batq_last_device_status() == 0
    return out.unflatten(1, (heads, d)).double().cpu(), *[R.gather(*x, list(range(pages)), n) for x in stored]


def _check(got, want, bound):
    far = (got - want).abs() / (bound + (want.abs() + bound) * 2.0 ** -8)
    assert far.max() <= 1, f"{int((far > 1).sum())} of {far.numel()} too far, worst {float(far.max()):.2f} of the bound"


@pytest.mark.parametrize("heads,kv_heads,d,rows", [(8, 2, 128, 1), (8, 2, 64, 5), (7, 1, 128, 3), (8, 2, 128, 50), (8, 2, 64, 40)])
@pytest.mark.parametrize("gap", [15, 20, 25, 30])
@pytest.mark.parametrize("size", [0.0, 2.0 ** -12, 2.0 ** -6])
@pytest.mark.parametrize("where", [0, 777])
def test_one_token_has_the_weight_and_no_values(batq, heads, kv_heads, d, rows, gap, size, where, copy_path):
    """A score `gap` binades above those of 4095 keys, whose values are of size 1; its own are `size` times that."""
    n = 4096
    g = torch.Generator().manual_seed(gap + where + rows)
    q = 0.5 * torch.randn(rows, heads, d, generator=g)
    q[..., 0] = 4.0
    k, v = 0.02 * torch.randn(n, kv_heads, d, generator=g), 1.0 + 0.3 * torch.randn(n, kv_heads, d, generator=g)
    k[:, :, 0] = 0.0
    k[where, :, 0] = gap * math.log(2.0) * d ** 0.5 / 4.0
    v[where] *= size
    q = q.bfloat16()
    got, kq, vq = _attend(batq, q, k, v, 64)
    _check(got, *_reference(q, kq, vq, d ** -0.5))


@pytest.mark.parametrize("d,rows", [(128, 1), (128, 50), (64, 1), (64, 50)])
@pytest.mark.parametrize("exponent", [-60, -30, 30, 60])
def test_all_values_tiny_or_huge(batq, d, rows, exponent, copy_path):
    g = torch.Generator().manual_seed(rows + exponent)
    q = torch.randn(rows, 8, d, generator=g).bfloat16()
    k, v = (torch.randn(512, 2, d, generator=g) for _ in range(2))
    got, kq, vq = _attend(batq, q, k, v.double() * 2.0 ** exponent, 32)
    want, bound = _reference(q, kq, vq * 2.0 ** -exponent, d ** -0.5)
    _check(got * 2.0 ** -exponent, want, bound)


def test_bad_tokens_of_a_prompt_leave_the_others(batq, copy_path):
    """A NaN and an infinity among a prompt's tokens: rows that do not see them come out as without them.  In the tiles
    of 128 tokens in front to the bit, in the bad token's own up to roundings."""
    heads, kv_heads, d, tokens = 8, 2, 64, 640
    a = Append(batq, tokens, heads, kv_heads, d, 16, rot=d, transform=True, clip=True, seed=12)
    slots = torch.arange(tokens)
    table = torch.arange(tokens // 16, dtype=torch.int32, device="cuda")[None].contiguous()
    starts, lens = torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), torch.tensor([tokens], dtype=torch.int32, device="cuda")
    x = a.x.cuda()
    bad = x.clone()
    bad[300, heads * d + 3] = math.nan                                      # a key
    bad[300, (heads + kv_heads) * d:(heads + kv_heads) * d + 32] = math.nan  # a block of values
    bad[560, heads * d + 70] = math.inf
    bad[560, (heads + kv_heads) * d + 1] = -math.inf
    outs = []
    for y in (x, bad):
        q_out = torch.empty(tokens, heads * d, dtype=torch.bfloat16, device="cuda")
        a.run(batq, x=y, q_out=q_out, slots=slots)
        out = torch.zeros_like(q_out)
        ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(a.cache, heads, tokens, 1, tokens, tokens))
        batq.batq_attention_kv_mxfp8(a.cache, q_out, out, lens, table, tokens, tokens, ws, q_starts=starts)
        assert batq.batq_last_device_status() == 0
        outs.append(out.float())
        if y is x:
            clean = [a.pool[2].clone(), a.pool[3].clone()]
    assert torch.equal(outs[0][:256], outs[1][:256])
    # weights are off by 2^-11 of themselves on both sides, their scores are the same
    most = R.values(*[b.cpu() for b in clean]).abs().max()
    assert ((outs[0] - outs[1])[256:300].abs().cpu() <= outs[0][256:300].abs().cpu() * 2.0 ** -7 + most * 2.0 ** -9).all()
