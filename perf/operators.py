"""What is timed of the 8-bit key/value cache: filling it and attending over it, over the sizes a server does that at.

Two operators.

  "append"     new tokens' keys and values go into a paged cache: the keys' position rotation, the keys' and the
               values' block transform and clip, MXFP8 (E4M3 codes, one E8M0 scale for each token, head and 32
               channels), stored at the tokens' slots; the queries of the same tokens are rotated and taken through
               the keys' dual transform P^-T, so that q' k'^T is q k^T.
  "attention"  softmax(scale q k^T) v over that cache through a page table, the sequences of a batch each with a
               length and a number of query rows of its own (one: decoding; several: checking a draft; many: a prompt
               or a chunk of one), grouped heads, causal from the sequence's end.

`run` computes them in torch (`own` false) or makes a user's calls of the library (`own` true).
"""
from __future__ import annotations

import math
import random

import torch

own = False

LLAMA8B = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}     # heads of the 4096 -> 6144 projection
QWEN2VL7B = {"q_heads": 28, "kv_heads": 4, "head_dim": 128}   # heads of the 3584 -> 4608 projection
NARROW = {"q_heads": 16, "kv_heads": 4, "head_dim": 64}       # a small model's


def _append(name, tokens, shape, page, padding=0, transform=True):
    return {"name": name, "op": "append", "tokens": tokens, "padding": padding, **shape, "page": page, "transform": transform}


def _attention(name, seqs, queries, context, shape, page, lengths="even", rows="even"):
    return {"name": name, "op": "attention", "seqs": seqs, "queries": queries, "context": context, "lengths": lengths,
            "rows": rows, **shape, "page": page}


def listed():
    return [
        # one user's next token: launch and latency
        _append("append_1", 1, LLAMA8B, 64),
        # a decode batch padded to a fixed size for a captured step
        _append("append_61_of_64", 64, QWEN2VL7B, 32, padding=3),
        # a chunk of a prompt, of no tile's size
        _append("append_509", 509, LLAMA8B, 16),
        # a long prompt with image tokens
        _append("append_8192", 8192, QWEN2VL7B, 64),
        # one user's next token after a short prompt
        _attention("decode_1_short", 1, 1, 67, LLAMA8B, 64),
        # a decode step of a small batch, lengths as they come, one slot of the batch empty
        _attention("decode_16", 16, 1, 4001, LLAMA8B, 64, lengths="ragged"),
        # one user deep in a long document
        _attention("decode_1_long", 1, 1, 131072, LLAMA8B, 64),
        # a busy server's decode step: bandwidth
        _attention("decode_128", 128, 1, 8192, QWEN2VL7B, 32, lengths="ragged"),
        # up to five drafted tokens to check for each of 24 users of a small model
        _attention("verify_24", 24, 5, 2500, NARROW, 16, lengths="ragged", rows="ragged"),
        # the prefill that the library's headline figure is quoted on
        _attention("prefill_2048", 1, 2048, 2048, LLAMA8B, 64),
        # a long prompt with image tokens: the largest pass
        _attention("prefill_8192", 1, 8192, 8192, QWEN2VL7B, 128),
        # a chunk of one user's prompt beside fifteen users who decode
        _attention("mixed_16", 16, 509, 4096, LLAMA8B, 64, lengths="ragged", rows="chunk"),
    ]


def draw(rng):
    def log(a, b):
        return min(b, max(a, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))

    shape = rng.choice([LLAMA8B, QWEN2VL7B, NARROW, {"q_heads": 8, "kv_heads": 8, "head_dim": 64},
                        {"q_heads": 12, "kv_heads": 1, "head_dim": 128}])
    page = rng.choice([16, 32, 64, 128])
    kind = rng.choice(["append", "decode", "decode", "verify", "prefill", "chunk"])
    if kind == "append":
        tokens = log(1, 8000)
        return {"op": "append", "tokens": tokens, "padding": rng.randint(0, min(3, tokens - 1)), **shape, "page": page,
                "transform": rng.random() < 0.75}
    case = {"op": "attention", **shape, "page": page, "lengths": rng.choice(["even", "ragged"])}
    if kind == "decode":
        seqs = log(1, 128)
        return {**case, "seqs": seqs, "queries": 1, "context": log(1, max(1, 600000 // seqs // shape["kv_heads"] * 2)), "rows": "even"}
    if kind == "verify":
        seqs = log(1, 32)
        return {**case, "seqs": seqs, "queries": rng.randint(2, 8), "context": log(16, 8000 // seqs * 8), "rows": "ragged"}
    if kind == "prefill":
        queries = log(17, 4096)
        return {**case, "seqs": 1, "queries": queries, "context": queries, "rows": "even", "lengths": "even"}
    seqs = log(2, 16)
    queries = log(17, 700)
    return {**case, "seqs": seqs, "queries": queries, "context": queries + log(1, 3000), "rows": rng.choice(["chunk", "ragged"])}


def _lengths(case):
    """Query rows and lengths of a case's sequences: the same for every seed."""
    r = random.Random(case["seqs"] * 1000003 + case["context"] * 17 + case["queries"])
    seqs, queries, context = case["seqs"], case["queries"], case["context"]
    rows = [queries] * seqs
    if case["rows"] == "ragged":
        rows = [queries] + [r.randint(1, queries) for _ in range(seqs - 1)]
    elif case["rows"] == "chunk":
        rows = [queries] + [1] * (seqs - 1)
    lens = [context] * seqs
    if case["lengths"] == "ragged":
        lens = [context] + [r.randint(min(context, n), context) for n in rows[1:]]
        if seqs >= 8:
            lens[seqs // 2], rows[seqs // 2] = 0, min(rows[seqs // 2], 1)   # an empty slot of the batch
    return rows, lens


def work(case):
    """Each input read once, each output written once; what a causal row does not see is not computed."""
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "append":
        t = case["tokens"] - case["padding"]
        token = 2 * d * (2 * hk + hq) + 2 * hk * (d + d // 32) + 2 * hq * d + 4 * d + 12
        flops = t * d * (hk * (3 + 24 + 4) + hk * (24 + 4) + hq * (3 + 24))
        return {"bytes": t * token, "flops": flops}
    rows, lens = _lengths(case)
    pairs = sum(sum(max(0, n - m + j + 1) for j in range(m)) for m, n in zip(rows, lens))
    read = sum(lens) * hk * 2 * (d + d // 32) + 4 * sum(-(-n // case["page"]) for n in lens)
    return {"bytes": read + 2 * sum(rows) * hq * d * 2, "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------------------------------------- inputs
def _mxfp8(y):
    """MXFP8 along the last axis, in y's precision: E4M3 codes and E8M0 bytes.  Scale exponent floor(log2 amax) - 8,
    elements to the nearest code (ties to even), saturating at 448."""
    b = y.unflatten(-1, (-1, 32))
    e = (torch.frexp(b.abs().amax(-1))[1] - 9).clamp(min=-127)
    e = torch.where(b.abs().amax(-1) > 0, e, torch.full_like(e, -127))
    u = torch.ldexp(b, -e.unsqueeze(-1)) if y.dtype == torch.float64 else b * torch.exp2(-e.unsqueeze(-1).float())
    step = torch.exp2((torch.frexp(u)[1] - 1).clamp(min=-6).to(y.dtype) - 3)
    u = (torch.round(u / step) * step).clamp(-448, 448)
    return u.flatten(-2).float().to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _factors(g, k):
    """A layer's transform: one 4 x 4 left factor, k right factors of 8 x 8, k clip ratios; and the dual's factors."""
    left = torch.eye(4) + 0.1 * torch.randn(1, 4, 4, generator=g)
    right = torch.eye(8) + 0.1 * torch.randn(k, 8, 8, generator=g)
    return left, right, 0.8 + 0.2 * torch.rand(k, generator=g)


def _rope_table(rows, d):
    """[rows, d]: the cosines of a position's d / 2 angles, then the sines."""
    angle = torch.arange(rows, device="cuda").double()[:, None] * torch.exp(
        torch.arange(0, d, 2, device="cuda").double() * (-math.log(500000.0) / d))
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    s = {"case": case}
    if own:
        from paper_2603_16590_b200 import binding as B
        s["B"] = B
    if case["op"] == "append":
        tokens = case["tokens"]
        pages = tokens // page + 3
        # q, k and v are column ranges of the projection's output; a few channels of the keys stand out
        qkv = torch.randn(tokens, (hq + 2 * hk) * d, device="cuda", generator=g)
        qkv[:, hq * d:(hq + hk) * d] *= 1 + 7.0 * (torch.rand(hk * d, device="cuda", generator=g) < 0.02)
        s["qkv"] = qkv.bfloat16()
        slots = torch.randperm(pages, device="cuda", generator=g)[:, None] * page + torch.arange(page, device="cuda")
        s["slots"] = slots.flatten()[3:3 + tokens].contiguous()
        if case["padding"]:
            s["slots"][tokens - case["padding"]:] = -1
        s["positions"] = torch.arange(tokens, device="cuda", dtype=torch.int32) + int(torch.randint(0, 1000, (1,), generator=host))
        s["rope"] = _rope_table(tokens + 1000, d)
        s["q_out"] = torch.zeros(tokens, hq * d, dtype=torch.bfloat16, device="cuda")
        fill = torch.randn(2, pages, hk, page, d, device="cuda", generator=g)
        s["factors"] = [_factors(host, d // 32) for _ in range(2)] if case["transform"] else None
    else:
        rows, lens = _lengths(case)
        counts = [-(-n // page) for n in lens]
        pages = sum(counts) + 2
        order = torch.randperm(pages, generator=host)[:sum(counts)]
        # entries behind a sequence's last page are not read: they hold page 0
        table = torch.zeros(len(lens), max(1, max(counts)), dtype=torch.int32)
        at = 0
        for i, n in enumerate(counts):
            table[i, :n] = order[at:at + n]
            at += n
        s["page_table"] = table.cuda()
        s["kv_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["q_starts"] = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32, device="cuda")
        s["max_q"], s["max_kv"] = max(rows), max(max(lens), 1)
        s["q"] = (2 * torch.randn(sum(rows), hq * d, device="cuda", generator=g)).bfloat16()
        s["out"] = torch.zeros(sum(rows), hq * d, dtype=torch.bfloat16, device="cuda")
        # tokens of different size, as keys and values of a model are
        fill = torch.randn(2, pages, hk, page, d, device="cuda", generator=g)
        fill *= torch.exp(0.5 * torch.randn(2, pages, hk, page, 1, device="cuda", generator=g))
    (s["k_codes"], s["k_scales"]), (s["v_codes"], s["v_scales"]) = _mxfp8(fill[0]), _mxfp8(fill[1])
    if own:
        s["cache"] = B.batq_kv_cache_create(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
        if case["op"] == "append":
            s["t_k"] = s["t_v"] = s["t_q"] = None
            if case["transform"]:
                (left, right, clip), (vleft, vright, vclip) = s["factors"]
                s["t_k"] = B.batq_transform_create(d, left.numpy(), right.numpy(), clip.numpy(), clip.numpy())
                s["t_v"] = B.batq_transform_create(d, vleft.numpy(), vright.numpy(), vclip.numpy(), vclip.numpy())
                s["t_q"] = B.batq_transform_create_dual(s["t_k"])
        else:
            n = B.batq_attention_kv_mxfp8_workspace_bytes(s["cache"], hq, s["q"].shape[0], case["seqs"], s["max_q"], s["max_kv"])
            s["workspace"] = B.aligned_workspace(n)
    elif case["op"] == "append" and case["transform"]:
        s["factors"] = [tuple(x.cuda() for x in f) for f in s["factors"]]
    return s


# ---------------------------------------------------------------------------------------------- the operators
def _rotated(x, cos, sin):
    """x [tokens, heads, d] in 64 bits, channel i with channel i + d / 2."""
    a, b = x.chunk(2, -1)
    cos, sin = cos[:, None], sin[:, None]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _transformed(x, left, right):
    """x P, block by block: L^T V R of each 32 channels as a 4 x 8 matrix."""
    v = x.unflatten(-1, (-1, 4, 8)) @ right.double()
    return (left.double().transpose(-1, -2) @ v).flatten(-3)


def _clipped(x, clip):
    b = x.unflatten(-1, (-1, 32))
    c = clip.double()[:, None]
    return torch.minimum(torch.maximum(b, c * b.amin(-1, keepdim=True)), c * b.amax(-1, keepdim=True)).flatten(-2)


def _append_plain(s):
    # in 64 bits: a code depends on which side of a border between two codes a value lies
    case = s["case"]
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    keep = s["slots"] >= 0
    x = s["qkv"][keep].double().unflatten(-1, (-1, d))
    cos, sin = s["rope"][s["positions"][keep].long()].double().chunk(2, -1)
    q, k, v = _rotated(x[:, :hq], cos, sin), _rotated(x[:, hq:hq + hk], cos, sin), x[:, hq + hk:]
    if s["factors"]:
        (left, right, clip), (vleft, vright, vclip) = s["factors"]
        q = _transformed(q, torch.linalg.inv(left.double()).transpose(-1, -2), torch.linalg.inv(right.double()).transpose(-1, -2))
        k = _clipped(_transformed(k, left, right), clip)
        v = _clipped(_transformed(v, vleft, vright), vclip)
    s["q_out"][keep] = q.flatten(1).bfloat16()
    at, off = s["slots"][keep] // page, s["slots"][keep] % page
    s["k_codes"][at, :, off], s["k_scales"][at, :, off] = _mxfp8(k)
    s["v_codes"][at, :, off], s["v_scales"][at, :, off] = _mxfp8(v)


def _values(codes, scales, table):
    """The pages of each sequence in a row, as values: [seqs, kv_heads, tokens, d]."""
    x = codes[table].view(torch.float8_e4m3fn).float().unflatten(-1, (-1, 32))
    x = torch.ldexp(x, scales[table].int().unsqueeze(-1) - 127).flatten(-2)
    return x.transpose(1, 2).flatten(2, 3)


def _attention_plain(s):
    case = s["case"]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    table, starts, lens = s["page_table"].long(), s["q_starts"].long(), s["kv_lens"].long()
    k, v = _values(s["k_codes"], s["k_scales"], table), _values(s["v_codes"], s["v_scales"], table)
    # [seqs, max_q] rows of q; rows behind a sequence's own are computed and dropped
    j = torch.arange(s["max_q"], device="cuda")
    count = starts[1:] - starts[:-1]
    have = j < count[:, None]
    row = (starts[:-1, None] + j).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[row].unflatten(-1, (hk, hq // hk, d)).permute(0, 2, 3, 1, 4)      # [seqs, hk, group, max_q, d]
    score = (q.flatten(2, 3) @ k.transpose(-1, -2)).unflatten(2, (hq // hk, -1)) * d ** -0.5
    last = lens[:, None] - count[:, None] + j                                            # the key a row sees last
    seen = torch.arange(k.shape[2], device="cuda") <= last[..., None]
    score = score.masked_fill(~seen[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    del score
    o = (p.flatten(2, 3) @ v).unflatten(2, (hq // hk, -1)) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    s["out"][row[have]] = o.permute(0, 3, 1, 2, 4).flatten(2)[have].bfloat16()


def run(s):
    case = s["case"]
    if case["op"] == "append":
        if own:
            B = s["B"]
            hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
            q, k, v = s["qkv"].split([hq * d, hk * d, hk * d], 1)
            B.batq_kv_append_mxfp8(s["cache"], s["t_k"], s["t_v"], k, v, s["slots"], positions=s["positions"], rope=s["rope"],
                                   t_q=s["t_q"], q=q, q_out=s["q_out"])
        else:
            _append_plain(s)
        # the cache as it stands: codes and scales as the values they stand for
        return {"q": s["q_out"], "k_codes": s["k_codes"].view(torch.float8_e4m3fn), "k_scales": s["k_scales"].view(torch.float8_e8m0fnu),
                "v_codes": s["v_codes"].view(torch.float8_e4m3fn), "v_scales": s["v_scales"].view(torch.float8_e8m0fnu)}
    if own:
        B = s["B"]
        B.batq_attention_kv_mxfp8(s["cache"], s["q"], s["out"], s["kv_lens"], s["page_table"], s["max_q"], s["max_kv"], s["workspace"],
                                  q_starts=s["q_starts"])
    else:
        _attention_plain(s)
    return {"out": s["out"]}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _nearest_e4m3(u):
    """The E4M3 value nearest to u, the even code where two are as near, from the list of all of them."""
    grid = torch.arange(127, dtype=torch.uint8, device=u.device).view(torch.float8_e4m3fn).double()
    middle = (grid[1:] + grid[:-1]) / 2
    a = u.abs().contiguous()
    low, high = torch.searchsorted(middle, a), torch.searchsorted(middle, a, right=True)   # they differ on a border
    return torch.copysign(grid[torch.where(low % 2 == 0, low, high)], u)


def _exact_cache(x, pool, codes, scales, slots):
    """x [tokens, heads, d] in 64 bits, into copies of a pool's codes and scales, as values."""
    codes = codes.view(torch.float8_e4m3fn).double()
    scales = torch.exp2(scales.double() - 127)
    blocks = x.reshape(*x.shape[:2], -1, 32)
    scale = torch.exp2(torch.floor(torch.log2(blocks.abs().amax(-1))) - 8)
    value = _nearest_e4m3(blocks / scale[..., None]).reshape(x.shape)
    page = pool["page"]
    for t, slot in enumerate(slots.tolist()):
        if slot >= 0:
            codes[slot // page, :, slot % page] = value[t]
            scales[slot // page, :, slot % page] = scale[t]
    return codes, scales


def exact(case, seed):
    s = prepare(case, seed)
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    if case["op"] == "append":
        x = s["qkv"].double().reshape(case["tokens"], hq + 2 * hk, d)
        angle = s["rope"][s["positions"].long()].double()
        turn = torch.complex(angle[:, :d // 2], angle[:, d // 2:])[:, None]
        z = torch.complex(x[:, :hq + hk, :d // 2].contiguous(), x[:, :hq + hk, d // 2:].contiguous()) * turn
        x[:, :hq + hk] = torch.cat([z.real, z.imag], -1)
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        if s["factors"]:
            def dense(f):
                return torch.block_diag(*[torch.kron(f[0][0].double(), r.double()) for r in f[1]]).cuda()

            def clip(y, f):
                y = y.reshape(*y.shape[:2], -1, 32)
                c = f[2].double().cuda()[:, None]
                return torch.clamp(y, c * y.min(-1, keepdim=True)[0], c * y.max(-1, keepdim=True)[0]).reshape(*y.shape[:2], d)

            p = dense(s["factors"][0])
            q = torch.linalg.solve(p, q.reshape(-1, d).T).T.reshape(q.shape)   # q P^-T
            k, v = clip(k @ p, s["factors"][0]), clip(v @ dense(s["factors"][1]), s["factors"][1])
        q = q.reshape(case["tokens"], -1) * (s["slots"] >= 0)[:, None]
        kc, ks = _exact_cache(k, case, s["k_codes"], s["k_scales"], s["slots"])
        vc, vs = _exact_cache(v, case, s["v_codes"], s["v_scales"], s["slots"])
        return {"q": q, "k_codes": kc, "k_scales": ks, "v_codes": vc, "v_scales": vs}
    rows, lens = _lengths(case)
    out = torch.zeros(sum(rows), hq, d, dtype=torch.float64, device="cuda")
    at = 0
    for i, (m, n) in enumerate(zip(rows, lens)):
        ids = s["page_table"][i, :-(-n // page)].long()
        for h in range(hk if n else 0):
            k, v = (x[ids, h].view(torch.float8_e4m3fn).double().reshape(-1, d // 32, 32)
                    * torch.exp2(y[ids, h].double() - 127).reshape(-1, d // 32, 1)
                    for x, y in ((s["k_codes"], s["k_scales"]), (s["v_codes"], s["v_scales"])))
            k, v = k.reshape(-1, d)[:n], v.reshape(-1, d)[:n]
            for e in range(h * (hq // hk), (h + 1) * (hq // hk)):
                for a in range(0, m, 2048):
                    b = min(m, a + 2048)
                    w = s["q"][at + a:at + b].double().reshape(b - a, hq, d)[:, e] @ k.T / math.sqrt(d)
                    hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - m + a, n - m + b, device="cuda")[:, None]
                    out[at + a:at + b, e] = torch.softmax(w.masked_fill(hidden, float("-inf")), -1) @ v
        at += m
    return {"out": out.reshape(sum(rows), hq * d)}
