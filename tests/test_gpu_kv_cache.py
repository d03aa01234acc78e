"""The 8-bit key/value cache on the GPU against its definition in 64 bits: the append, the attention, both in a row."""
import math

import pytest
import torch

import kv_reference as R
from paper_2603_16590_b200 import synth

pytestmark = pytest.mark.gpu
ERR_INDEX, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 9, 1, 2, 3, 4, 5


def _refused(batq, status, call):
    with pytest.raises(batq.BatqError) as e:
        call()
    assert e.value.status == status


def _pool(pages, heads, page, d, fill_code=0x7F, fill_scale=255):
    """Buffers full of NaN codes and NaN scales: whatever is read beyond what was written shows."""
    return [torch.full((pages, heads, page, last), v, dtype=torch.uint8, device="cuda")
            for last, v in ((d, fill_code), (d // 32, fill_scale)) * 2]


# ------------------------------------------------------------------------------------------------ attention
class Batch:
    """A filled cache with a page table: pages in a random order, everything behind a sequence's last key is NaN."""

    def __init__(self, batq, heads, kv_heads, d, page, rows, lens, seed=0, extra_q=0, spread=0.5, gain=2.0):
        g = torch.Generator().manual_seed(seed * 7919 + sum(lens) + page)
        counts = [-(-n // page) for n in lens]
        pages = sum(counts) + 3
        order = (torch.randperm(pages - 1, generator=g) + 1)[:sum(counts)].tolist()
        self.pages, at = [], 0
        for c in counts:
            self.pages.append(order[at:at + c])
            at += c
        kc, ks, vc, vs = (x.cpu() for x in _pool(pages, kv_heads, page, d))
        for codes, scales in ((kc, ks), (vc, vs)):
            x = torch.randn(pages, kv_heads, page, d, generator=g) * torch.exp(spread * torch.randn(pages, kv_heads, page, 1, generator=g))
            x = x * torch.exp(spread * torch.randn(1, kv_heads, 1, d // 32, generator=g)).repeat_interleave(32, -1)
            c, s = R.mxfp8(x.double())
            for i, n in enumerate(lens):
                for j, pg in enumerate(self.pages[i]):
                    m = min(page, n - j * page)
                    codes[pg, :, :m], scales[pg, :, :m] = c[pg, :, :m], s[pg, :, :m]
        self.k, self.v = (kc, ks), (vc, vs)
        self.buffers = [x.cuda() for x in (kc, ks, vc, vs)]
        self.cache = batq.batq_kv_cache_create(*self.buffers)
        width = max(1, max(counts))
        table = torch.full((len(lens), width), 1 << 30, dtype=torch.int32)   # behind the last page: not to be read
        for i, p in enumerate(self.pages):
            table[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
        self.table = table.cuda()
        self.rows, self.lens, self.heads, self.d = rows, lens, heads, d
        total = sum(rows) + extra_q
        self.q = (gain * torch.randn(total, heads, d, generator=g)).bfloat16()
        self.starts = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32).cuda()
        self.kv_lens = torch.tensor(lens, dtype=torch.int32).cuda()

    def run(self, batq, causal=True, max_q=None, max_kv=None, scale=None, use_starts=True, lse=True, q=None, out=None, workspace=None):
        q = self.q.cuda().flatten(1) if q is None else q
        out = torch.full((q.shape[0], self.heads * self.d), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        lse = torch.full((q.shape[0], self.heads), 5.0, device="cuda") if lse else None
        max_q, max_kv = max(self.rows) if max_q is None else max_q, max(max(self.lens), 1) if max_kv is None else max_kv
        n = batq.batq_attention_kv_mxfp8_workspace_bytes(self.cache, self.heads, q.shape[0], len(self.lens), max_q, max_kv)
        if workspace is None:
            workspace = batq.aligned_workspace(n)
            workspace.fill_(0xFF)
        batq.batq_attention_kv_mxfp8(self.cache, q, out, self.kv_lens, self.table, max_q, max_kv, workspace,
                                     q_starts=self.starts if use_starts else None, scale=scale, causal=causal, lse=lse)
        assert batq.batq_last_device_status() == 0
        return out.unflatten(1, (self.heads, self.d)), lse

    def check(self, out, lse, causal=True, scale=None, hidden=None):
        scale = self.d ** -0.5 if scale is None else scale
        n = sum(self.rows)
        want, wlse, bound = R.attention(self.q[:n], self.k, self.v, self.rows, self.lens, self.pages, scale, causal, hidden)
        got = out[:n].double().cpu()
        limit = bound + (want.abs() + bound) * 2.0 ** -8 + 2.0 ** -133
        far = (got - want).abs() > limit
        assert not torch.isnan(got).any() and not far.any(), (
            f"{int(far.sum())} of {far.numel()} too far, worst {float(((got - want).abs() / limit).max()):.2f} of the bound")
        if lse is not None:
            got = lse[:n].double().cpu()
            assert torch.equal(torch.isinf(got), torch.isinf(wlse))
            fine = ~torch.isinf(wlse)
            # scores as in the bound above (their largest error), the logarithm and one rounding to fp32
            rel = 2.0 ** -16 + wlse[fine].abs() * 2.0 ** -22
            k = [R.gather(*self.k, p, m) for p, m in zip(self.pages, self.lens)]
            big = max([float(x.norm(dim=-1).max()) for x in k if x.numel()] + [0.0]) * float(self.q.double().norm(dim=-1).max()) * abs(scale)
            assert ((got[fine] - wlse[fine]).abs() <= rel + big * (self.d + 8) * 2.0 ** -24).all()
        assert (out[n:] == 7.0).all() and (lse is None or (lse[n:] == 5.0).all())


@pytest.fixture(params=[1, 2], ids=["codes", "copy"])
def copy_path(batq, request):
    """Prompts from the codes, or from the f16 copy in the workspace, whatever the call's sizes would choose."""
    batq.batq_debug_force_attention_copy(request.param)
    yield request.param
    batq.batq_debug_force_attention_copy(0)


HEADS = [(32, 8, 128), (28, 4, 128), (3, 3, 128), (12, 1, 128), (16, 4, 64), (5, 5, 64), (20, 2, 64)]


@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decode_lengths(batq, heads, kv_heads, d, page):
    """One row per sequence; lengths of zero, one, and around tiles and pages."""
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 300, 0]
    b = Batch(batq, heads, kv_heads, d, page, [1] * len(lens), lens, seed=1)
    b.check(*b.run(batq, use_starts=False))


@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 128), (28, 4, 128), (12, 1, 128), (16, 4, 64)])
@pytest.mark.parametrize("lens", [[1], [67], [1000], [5003], [2049, 3, 0, 1500]])
def test_decode_long(batq, heads, kv_heads, d, lens):
    b = Batch(batq, heads, kv_heads, d, 64, [1] * len(lens), lens, seed=2)
    b.check(*b.run(batq))


@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 128), (28, 4, 128), (2, 2, 128), (16, 4, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_several_rows(batq, heads, kv_heads, d, causal):
    """Drafts and short chunks; more rows than keys leave the first ones empty; rows behind the last sequence stay."""
    rows, lens = [2, 5, 1, 0, 3, 9, 4, 7], [2, 40, 33, 17, 1, 1200, 0, 3]
    b = Batch(batq, heads, kv_heads, d, 32, rows, lens, seed=3, extra_q=4)
    b.check(*b.run(batq, causal=causal), causal=causal)


@pytest.mark.parametrize("heads,kv_heads,d,page", [(32, 8, 128, 64), (28, 4, 128, 16), (12, 1, 128, 128), (16, 4, 64, 32), (3, 3, 64, 16)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,lens", [([129], [129]), ([1, 77, 300, 1], [513, 78, 300, 1]), ([64], [1500]), ([200, 31], [150, 31]),
                                       ([12, 8, 3], [700, 9, 40])])
def test_prompts(batq, heads, kv_heads, d, page, causal, rows, lens, copy_path):
    """Whole prompts, chunks behind a context, more rows than keys."""
    b = Batch(batq, heads, kv_heads, d, page, rows, lens, seed=4, extra_q=2)
    b.check(*b.run(batq, causal=causal), causal=causal)


def test_more_sequences_than_one_launch(batq):
    """1500 short sequences, some empty, some without rows; and without row starts."""
    lens = [(7 * i) % 70 for i in range(1500)]
    b = Batch(batq, 4, 2, 64, 16, [(i % 5 != 3) + (i % 11 == 0) for i in range(1500)], lens, seed=18)
    b.check(*b.run(batq))
    b = Batch(batq, 4, 2, 64, 16, [1] * 1500, lens, seed=19)
    b.check(*b.run(batq, use_starts=False))


def test_prompt_beside_decoding(batq, copy_path):
    rows, lens = [1] * 6 + [173] + [1] * 3, [900, 3, 64, 65, 0, 511, 700, 1, 1025, 33]
    b = Batch(batq, 32, 8, 128, 64, rows, lens, seed=5)
    b.check(*b.run(batq))


@pytest.mark.parametrize("rows", [[1, 1, 1], [40, 1, 19]])
def test_bounds_may_be_larger_than_the_batch(batq, rows, copy_path):
    """max_q and max_kv size the grid only; a captured call meets other lengths within them."""
    b = Batch(batq, 32, 8, 128, 64, rows, [700, 64, 19], seed=6)
    b.check(*b.run(batq, max_q=300, max_kv=20000))


def test_where_keys_are_widened_once(batq):
    """The copy is in the workspace of large prompts, not of small or of huge ones (max_kv is a bound: the grid's alone)."""
    b = Batch(batq, 32, 8, 128, 64, [150, 1, 77], [700, 64, 77], seed=20)

    def copied(*sizes):
        """Bytes of workspace beyond what the call wants without a copy."""
        batq.batq_debug_force_attention_copy(1)
        least = batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 32, *sizes)
        batq.batq_debug_force_attention_copy(0)
        return batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 32, *sizes) - least

    copy = lambda seqs, max_kv: seqs * 8 * -(-max_kv // 128) * 65536  # noqa: E731
    assert copied(2048, 1, 2048, 2048) >= copy(1, 2048)
    assert copied(8 * 512, 8, 512, 8192) >= copy(8, 8192)
    assert copied(64, 1, 64, 8192) == copied(100000, 1, 100000, 200000) == copied(228, 3, 150, 200000) == 0
    b.check(*b.run(batq, max_kv=200000))


@pytest.mark.parametrize("rows", [1, 5, 70])
def test_no_keys_at_all(batq, rows):
    b = Batch(batq, 8, 2, 64, 16, [rows, rows], [0, 0], seed=21)
    for max_kv in (0, 1, 500):
        out, lse = b.run(batq, max_kv=max_kv)
        assert (out == 0).all() and torch.isinf(lse).all() and (lse < 0).all()


def test_lengths_beyond_the_bounds_are_not_looked_at(batq):
    b = Batch(batq, 8, 2, 128, 32, [1, 1], [100, 90], seed=7)
    got, _ = b.run(batq, max_kv=64)
    b.lens = [64, 64]
    b.check(got, None)
    b = Batch(batq, 8, 2, 128, 32, [3, 2], [50, 20], seed=8)
    b.kv_lens[0] = 1 << 29          # longer than the page table: two pages of it are there
    b.table = b.table[:, :2].contiguous()
    got, _ = b.run(batq, max_kv=1 << 30)
    # rows see what a length of 64 would show them; the last 14 keys are not finite here, so only the other sequence counts
    b.rows, b.q, b.lens, b.pages = b.rows[1:], b.q[3:], b.lens[1:], b.pages[1:]
    b.check(got[3:], None)


def test_scale_and_gain(batq, copy_path):
    """A scale of the caller's; sharp and flat distributions; queries and values of very different sizes."""
    for scale, gain in ((1.0, 1.0), (0.01, 30.0), (-0.2, 1.0), (0.0, 1.0)):
        b = Batch(batq, 16, 4, 64, 16, [1, 6], [300, 90], seed=9, gain=gain)
        b.check(*b.run(batq, scale=scale), scale=scale)
    for gain in (1e-30, 1e-6, 1e6):
        b = Batch(batq, 32, 8, 128, 64, [1, 30], [200, 64], seed=10, gain=gain)
        b.check(*b.run(batq, scale=1.0 / gain / 11), scale=1.0 / gain / 11)


@pytest.mark.parametrize("rows", [1, 50])
def test_value_scales_far_apart(batq, rows, copy_path):
    """A token with huge values and next to no weight, a token with all the weight and tiny values, blocks of zeros."""
    b = Batch(batq, 8, 2, 128, 32, [rows], [400], seed=11, spread=0.1)
    kc, ks = b.k
    vc, vs = b.v
    p = b.pages[0]
    vs[p[2], :, 5] += 20                       # values 2^20 times as large
    vs[p[5]] -= 14
    vc[p[7]] = 0                               # a page of zeros, with the least scale
    vs[p[7]] = 0
    vs[p[9], :, :, 1] -= 12                    # one block of channels much smaller
    b.buffers[2].copy_(vc)
    b.buffers[3].copy_(vs)
    b.check(*b.run(batq))


def test_strides_and_in_between_columns(batq, copy_path):
    """q and out as column ranges of wider tensors; what lies beside them stays."""
    b = Batch(batq, 8, 2, 128, 32, [1, 3, 40], [77, 40, 100], seed=12)
    wide = torch.full((44, 8 * 128 + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 1024] = b.q.cuda().flatten(1)
    out = torch.full((44, 8 * 128 + 40), 7.0, dtype=torch.bfloat16, device="cuda")
    b.run(batq, q=wide[:, 8:8 + 1024], out=out[:, 16:16 + 1024])
    b.check(out[:, 16:16 + 1024].unflatten(1, (8, 128)), None)
    assert (out[:, :16] == 7).all() and (out[:, 16 + 1024:] == 7).all()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("rows", [1, 45])
def test_bad_pages_are_left_out_and_reported(batq, page, rows, copy_path):
    b = Batch(batq, 8, 4, 64, page, [rows, rows], [200, 150], seed=13)
    hidden = [torch.zeros(200, dtype=torch.bool), torch.zeros(150, dtype=torch.bool)]
    for seq, at, bad in ((0, 1, -1), (1, 0, b.buffers[0].shape[0]), (1, 1, 1 << 30)):
        b.table[seq, at] = bad
        hidden[seq][at * page:(at + 1) * page] = True
    q, out = b.q.cuda().flatten(1), torch.full((2 * rows, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 8, 2 * rows, 2, rows, 200))
    batq.batq_attention_kv_mxfp8(b.cache, q, out, b.kv_lens, b.table, rows, 200, ws, q_starts=b.starts)
    assert batq.batq_last_device_status() == ERR_INDEX
    assert batq.batq_last_device_status() == 0
    b.check(out.unflatten(1, (8, 64)), None, hidden=hidden)


def test_row_starts_out_of_order_stay_inside(batq):
    """Nonsense in q_starts reads and writes nothing outside q and out; rows of sound sequences come out right."""
    b = Batch(batq, 8, 2, 128, 32, [2, 3, 2], [40, 50, 60], seed=14)
    guard = torch.full((7 + 64, 1024), 7.0, dtype=torch.bfloat16, device="cuda")
    for starts in ([-5, 2, 1 << 30, 7], [5, 3, 7, 100], [1 << 30, -(1 << 31), 5, 7]):
        s = torch.tensor(starts, dtype=torch.int32, device="cuda")
        ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 8, 7, 3, 3, 60))
        batq.batq_attention_kv_mxfp8(b.cache, b.q.cuda().flatten(1), guard[:7], b.kv_lens, b.table, 3, 60, ws, q_starts=s)
        assert batq.batq_last_device_status() == 0
        assert (guard[7:] == 7).all()


@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [3, 1, 70, 2]])
def test_captured_and_replayed_with_other_lengths(batq, rows, copy_path):
    """One capture, replayed after the lengths, the page table and the queries have changed; on a stream of its own."""
    b = Batch(batq, 32, 8, 128, 64, rows, [600, 40, 130, 2000], seed=15)
    q, out, lse = b.q.cuda().flatten(1), torch.full((sum(rows), 4096), 7.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(sum(rows), 32, device="cuda")
    ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 32, sum(rows), 4, max(rows), 2000))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        batq.batq_attention_kv_mxfp8(b.cache, q, out, b.kv_lens, b.table, max(rows), 2000, ws, q_starts=b.starts, lse=lse)
    for lens in ([600, 40, 130, 2000], [1, 40, 99, 1999], [600, 0, 130, 64]):
        b.lens = lens
        b.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        b.q = (b.q.double() * 0.9).bfloat16()
        q.copy_(b.q.flatten(1))
        ws.fill_(0xFF)
        graph.replay()
        assert batq.batq_last_device_status() == 0
        b.check(out.unflatten(1, (32, 128)), lse)


def test_same_bits_again_and_on_two_streams(batq, copy_path):
    """Repeated and concurrent calls give the same bits."""
    b = Batch(batq, 28, 4, 128, 64, [1, 1, 40, 2], [5000, 100, 300, 900], seed=16)
    first, lse = b.run(batq)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            out = torch.full((44, 3584), 7.0, dtype=torch.bfloat16, device="cuda")
            n = batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 28, 44, 4, 40, 5000)
            ws = batq.aligned_workspace(n)
            q = b.q.cuda().flatten(1)
            for _ in range(3):
                batq.batq_attention_kv_mxfp8(b.cache, q, out, b.kv_lens, b.table, 40, 5000, ws, q_starts=b.starts)
            got.append((out, ws, q))
    torch.cuda.synchronize()
    for out, _, _ in got:
        assert torch.equal(out.unflatten(1, (28, 128)).view(torch.int16), first.view(torch.int16))


def test_attention_refuses(batq):
    b = Batch(batq, 8, 2, 128, 32, [2, 3], [40, 50], seed=17)
    q, out = b.q.cuda().flatten(1), torch.zeros(5, 1024, dtype=torch.bfloat16, device="cuda")
    call = lambda **k: batq.batq_attention_kv_mxfp8(  # noqa: E731
        k.pop("cache", b.cache), k.pop("q", q), k.pop("out", out), k.pop("kv_lens", b.kv_lens), k.pop("table", b.table), k.pop("max_q", 3),
        k.pop("max_kv", 50), k.pop("ws", None), q_starts=k.pop("starts", b.starts), **k)
    big = batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, 8, 5, 2, 3, 1 << 20)
    assert big > 0
    _refused(batq, SHAPE, lambda: call(starts=None))                     # one row per sequence: 5 rows, 2 sequences
    _refused(batq, SHAPE, lambda: call(max_q=0))
    _refused(batq, SHAPE, lambda: call(max_kv=-1))
    _refused(batq, SHAPE, lambda: call(max_kv=(1 << 30) + 1))
    _refused(batq, SHAPE, lambda: call(scale=math.nan))
    _refused(batq, SHAPE, lambda: call(q=q[:, :384], out=out[:, :384]))                    # 3 heads over 2
    _refused(batq, SHAPE, lambda: call(q=torch.zeros(1024, dtype=torch.bfloat16, device="cuda").expand(5, 1024)))
    _refused(batq, ALIGN, lambda: call(q=torch.zeros(5, 1028, dtype=torch.bfloat16, device="cuda")[:, :1024]))
    _refused(batq, ALIGN, lambda: call(out=torch.zeros(5, 1032, dtype=torch.bfloat16, device="cuda")[:, 4:1028]))
    _refused(batq, NULL, lambda: call(max_kv=1 << 20))                   # needs a workspace
    _refused(batq, WORKSPACE, lambda: call(max_kv=1 << 20, ws=batq.aligned_workspace(big)[:big - 256]))
    _refused(batq, ALIGN, lambda: call(max_kv=1 << 20, ws=batq.aligned_workspace(big + 256)[16:]))
    empty = torch.zeros(0, 1024, dtype=torch.bfloat16, device="cuda")
    call(q=empty, out=empty, kv_lens=b.kv_lens[:0], table=b.table[:0], starts=None)     # nothing to do
    assert batq.batq_last_device_status() == 0 and (out == 0).all()


# ------------------------------------------------------------------------------------------------ append
def _table(rows, rot, seed=0):
    angle = torch.arange(rows).double()[:, None] * torch.exp(torch.arange(0, rot, 2).double() * (-math.log(10000.0) / rot))
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _transforms(batq, d, gr, gc, seed, clip=True):
    t = synth.make_transform(d, seed, "naive", clip=clip, gr=gr, gc=gc)
    return t, batq.batq_transform_create(d, t.left, t.right, t.clip_lo, t.clip_hi, gr=gr, gc=gc)


def _check_codes(got_codes, got_scales, y, bound):
    """Codes and scale bytes of y (fp64): as the definition has them, but for values that the fp32 error `bound` takes across a border."""
    codes, scales = R.mxfp8(y)
    amax = y.abs().unflatten(-1, (-1, 32)).amax(-1)
    bmax = bound.unflatten(-1, (-1, 32)).amax(-1)
    other = got_scales != scales
    if other.any():
        near = torch.exp2(torch.round(torch.log2(amax[other])))
        assert ((amax[other] - near).abs() <= bmax[other]).all()
    u = y.abs() / torch.exp2(scales.double() - 127).repeat_interleave(32, -1)
    du = bound / torch.exp2(scales.double() - 127).repeat_interleave(32, -1)
    wrong = (got_codes != codes) & ~other.repeat_interleave(32, -1)
    if wrong.any():
        a = u[wrong].contiguous()
        i = torch.searchsorted(R.MIDDLE, a).clamp(max=len(R.MIDDLE) - 1)
        dist = torch.minimum((R.MIDDLE[i] - a).abs(), (R.MIDDLE[(i - 1).clamp(min=0)] - a).abs())
        zero = (got_codes[wrong] & 127) + (codes[wrong] & 127) == 0      # a zero of the other sign
        assert ((dist <= du[wrong]) | (zero & (a <= du[wrong]))).all()
        assert (((got_codes[wrong] & 127).int() - (codes[wrong] & 127).int()).abs() <= 1).all()
    assert wrong.double().mean() <= 1e-3 and other.double().mean() <= 1e-3


class Append:
    def __init__(self, batq, tokens, heads, kv_heads, d, page, rot=None, gr=4, gc=8, transform=True, clip=True, seed=0, positions=True,
                 padding=(), gain=8.0):
        g = torch.Generator().manual_seed(1000 + seed + tokens)
        self.tokens, self.heads, self.kv_heads, self.d, self.page = tokens, heads, kv_heads, d, page
        width = (heads + 2 * kv_heads) * d
        x = torch.randn(tokens, width, generator=g)
        x = x * (1 + (gain - 1) * (torch.rand(width, generator=g) < 0.03))
        self.x = x.bfloat16()
        pages = tokens // page + 3
        slots = (torch.randperm(pages, generator=g)[:, None] * page + torch.arange(page)).flatten()[5:5 + tokens].contiguous()
        for i in padding:
            slots[i] = -1 - i
        self.slots = slots
        self.rot = rot
        self.table = _table(tokens + 300, rot) if rot else None
        self.positions = torch.randint(0, tokens + 300, (tokens,), generator=g).int() if positions and rot else None
        self.pool = _pool(pages, kv_heads, page, d, fill_code=0x33, fill_scale=99)
        self.cache = batq.batq_kv_cache_create(*self.pool)
        self.tk = self.tv = self.tq = self.k_t = self.v_t = None
        if transform:
            self.k_t, self.tk = _transforms(batq, d, gr, gc, 50 + seed, clip)
            self.v_t, self.tv = _transforms(batq, d, gr, gc, 60 + seed, clip)
            self.tq = batq.batq_transform_create_dual(self.tk)

    def split(self, x):
        return x.split([self.heads * self.d, self.kv_heads * self.d, self.kv_heads * self.d], 1)

    def run(self, batq, x=None, q_out=None, slots=None, positions=None, with_q=True):
        x = self.x.cuda() if x is None else x
        q, k, v = self.split(x)
        self.q_out = torch.full((self.tokens, self.heads * self.d), 7.0, dtype=torch.bfloat16, device="cuda") if q_out is None else q_out
        positions = self.positions if positions is None else positions
        batq.batq_kv_append_mxfp8(self.cache, self.tk, self.tv, k, v, (self.slots if slots is None else slots).cuda(),
                                  positions=None if positions is None else positions.cuda(), rope=None if self.table is None else self.table.cuda(),
                                  t_q=self.tq if with_q else None, q=q if with_q else None, q_out=self.q_out if with_q else None)

    def want(self):
        """q, k, v after rotation, transform and clip, in 64 bits, and the bounds on the fp32 kernel's error: each is
        sum_i |x_i| |P_ij| over the 32 channels of a block with |x| the rotation's |a cos| + |b sin|, and at most
        2 (rotation) + 8 + 4 (the factors' sums; 32 + 1 where the matrix is one factor) + 2 (clip, scale) roundings of 2^-24."""
        x = self.x.double().unflatten(1, (-1, self.d))
        parts = list(x.split([self.heads, self.kv_heads, self.kv_heads], 1))
        mags = [p.abs() for p in parts]
        if self.rot:
            rows = self.table[self.positions.long() if self.positions is not None else torch.arange(self.tokens)]
            for i in (0, 1):
                a, b = parts[i].abs()[..., :self.rot // 2], parts[i].abs()[..., self.rot // 2:self.rot]
                c, s = rows.double().abs()[:, None].chunk(2, -1)
                mags[i] = torch.cat([a * c + b * s, b * c + a * s, parts[i].abs()[..., self.rot:]], -1)
                parts[i] = R.rotate(parts[i], rows)
        k = self.d // 32
        for i, t in ((1, self.k_t), (2, self.v_t)):
            if t is not None:
                p = R.dense(t.left, t.right, k)
                parts[i] = R.transform(parts[i], p)
                mags[i] = R.transform(mags[i], p.abs())
                if t.clip_lo is not None:
                    parts[i] = R.clip(parts[i], t.clip_lo, t.clip_hi)
                    mags[i] = mags[i].unflatten(-1, (-1, 32)).amax(-1, keepdim=True).expand(*mags[i].shape[:-1], k, 32).flatten(-2)
                if i == 1 and self.tq is not None:
                    inv = torch.linalg.inv(p).transpose(-1, -2)
                    parts[0], mags[0] = R.transform(parts[0], inv), R.transform(mags[0], inv.abs() * 1.0)
        return parts, [m * 36 * 2.0 ** -24 for m in mags]

    def check(self):
        (q, k, v), (bq, bk, bv) = self.want()
        keep = self.slots >= 0
        kc, ks, vc, vs = (x.cpu() for x in self.pool)
        at, off = self.slots[keep] // self.page, self.slots[keep] % self.page
        for codes, scales, y, b in ((kc, ks, k, bk), (vc, vs, v, bv)):
            _check_codes(codes[at, :, off], scales[at, :, off], y[keep], b[keep])
            codes[at, :, off], scales[at, :, off] = 0x33, 99
            assert (codes == 0x33).all() and (scales == 99).all()        # nothing else was written
        got = self.q_out.unflatten(1, (self.heads, self.d)).double().cpu()
        assert ((got - q)[keep].abs() <= (q.abs() * 2.0 ** -8 + bq * 1.01 + 2.0 ** -133)[keep]).all()
        assert (got[~keep] == 7.0).all()


@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 128), (28, 4, 128), (16, 4, 64), (3, 1, 128), (5, 5, 64)])
@pytest.mark.parametrize("tokens,page", [(1, 64), (2, 16), (37, 32), (130, 128), (509, 16)])
def test_append(batq, heads, kv_heads, d, tokens, page):
    a = Append(batq, tokens, heads, kv_heads, d, page, rot=d)
    a.run(batq)
    assert batq.batq_last_device_status() == 0
    a.check()


@pytest.mark.parametrize("gr,gc", [(1, 32), (2, 16), (4, 8), (8, 4), (16, 2), (32, 1)])
@pytest.mark.parametrize("clip", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_append_factor_sizes(batq, gr, gc, clip, d):
    a = Append(batq, 70, 8, 2, d, 32, rot=d, gr=gr, gc=gc, clip=clip, seed=2)
    a.run(batq)
    a.check()


@pytest.mark.parametrize("d,rot", [(128, 16), (128, 32), (128, 48), (128, 64), (128, 112), (64, 16), (64, 48), (128, None)])
@pytest.mark.parametrize("transform", [True, False])
def test_append_rotations(batq, d, rot, transform):
    """Part of a head rotated, at every kind of partner distance; none rotated; with and without a transform."""
    a = Append(batq, 65, 12, 3, d, 64, rot=rot, transform=transform, seed=3)
    a.run(batq)
    a.check()


def test_append_one_table_row_per_token(batq):
    a = Append(batq, 40, 8, 2, 128, 32, rot=128, positions=False, seed=4)
    a.run(batq)
    a.check()


def test_append_padding_rows(batq):
    a = Append(batq, 45, 28, 4, 128, 32, rot=128, padding=(0, 7, 8, 43, 44), seed=5)
    a.run(batq)
    assert batq.batq_last_device_status() == 0
    a.check()


def test_append_bad_indexes_are_left_out_and_reported(batq):
    a = Append(batq, 30, 8, 2, 64, 16, rot=64, seed=6)
    slots, positions = a.slots.clone(), a.positions.clone()
    n = a.pool[0].shape[0] * 16
    slots[3], slots[9], positions[12], positions[20] = n, 1 << 40, -1, a.table.shape[0]
    a.run(batq, slots=slots, positions=positions)
    assert batq.batq_last_device_status() == ERR_INDEX
    assert batq.batq_last_device_status() == 0
    a.slots[[3, 9, 12, 20]] = -1
    a.check()


def test_append_queries_in_place_and_transforms_of_different_sizes(batq):
    a = Append(batq, 50, 8, 2, 128, 64, rot=128, seed=7)
    x = a.x.cuda()
    a.run(batq, x=x, q_out=a.split(x)[0])
    a.check()
    b = Append(batq, 50, 8, 2, 128, 64, rot=128, seed=8)
    b.v_t, b.tv = _transforms(batq, 128, 8, 4, 77)
    b.run(batq)
    b.check()
    b = Append(batq, 50, 8, 2, 128, 64, rot=128, seed=9)
    b.v_t = b.tv = None
    b.run(batq)
    b.check()


def test_append_is_the_quantiser_where_nothing_is_rotated(batq):
    """Without a rotation the cache holds batq_quantize_act_mxfp8's codes of the heads' rows."""
    a = Append(batq, 200, 4, 4, 128, 32, rot=None, seed=10)
    a.run(batq)
    k = a.split(a.x.cuda())[1].contiguous().view(-1, 128)
    codes = torch.empty(800, 128, dtype=torch.uint8, device="cuda")
    scales = torch.empty(800, 4, dtype=torch.uint8, device="cuda")
    batq.batq_quantize_act_mxfp8(a.tk, k, codes, scales, 0)
    at, off = (a.slots // 32).cuda(), (a.slots % 32).cuda()
    assert (a.pool[0][at, :, off].view(-1, 128) != codes).double().mean() <= 1e-5
    assert (a.pool[1][at, :, off].view(-1, 4) != scales).double().mean() <= 1e-5


@pytest.mark.parametrize("transform,clip", [(False, False), (True, False), (True, True)])
def test_append_stores_no_nan(batq, transform, clip):
    """A NaN (one element, a whole block) or an infinity: finite codes there, the other tokens as without it, and an
    attention whose rows that do not see the token are the same."""
    a = Append(batq, 60, 8, 2, 64, 16, rot=64, transform=transform, clip=clip, seed=12)
    a.run(batq)
    clean = [x.clone() for x in a.pool]
    x = a.x.cuda().clone()
    x[40, 8 * 64 + 3] = math.nan              # a key
    x[40, 10 * 64:10 * 64 + 32] = math.nan    # a block of values
    x[40, 11 * 64 + 40] = math.nan
    x[50, 8 * 64 + 70] = math.inf
    x[50, 9 * 64 + 1] = -math.inf
    a.run(batq, x=x)
    others = [i for i in range(60) if i not in (40, 50)]
    at, off = (a.slots // 16).cuda(), (a.slots % 16).cuda()
    for before, now in zip(clean, a.pool):
        assert torch.equal(before[at, :, off][others], now[at, :, off][others])
    for codes in (a.pool[0], a.pool[2]):
        assert ((codes & 0x7F) != 0x7F).all()
    table = torch.arange(a.pool[0].shape[0], dtype=torch.int32, device="cuda")[None].contiguous()
    rows = torch.zeros(2, dtype=torch.int32, device="cuda")
    # one sequence over the pool in slot order: the rows in front of the bad tokens' slots see none of them
    first = int(min(a.slots[40], a.slots[50]))
    n = table.shape[1] * 16
    qs = torch.randn(n, 8 * 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    outs = []
    for pool in (clean, a.pool):
        cache = batq.batq_kv_cache_create(*[p.clone() for p in pool])
        out = torch.zeros(n, 8 * 64, dtype=torch.bfloat16, device="cuda")
        ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(cache, 8, n, 1, n, n))
        rows[1] = n
        batq.batq_attention_kv_mxfp8(cache, qs, out, torch.tensor([n], dtype=torch.int32, device="cuda"), table, n, n, ws, q_starts=rows)
        outs.append(out)
    assert batq.batq_last_device_status() == 0
    assert torch.isfinite(outs[1][:first].float()).all()
    if int(a.slots[50]) > first + 128 or int(a.slots[50]) // 128 != first // 128:   # (an infinity's scale is felt within its tile)
        assert torch.equal(outs[0][:first], outs[1][:first])


def test_append_refuses(batq):
    a = Append(batq, 10, 8, 2, 128, 32, rot=128, seed=11)
    x = a.x.cuda()
    q, k, v = a.split(x)
    slots, rope, pos = a.slots.cuda(), a.table.cuda(), a.positions.cuda()
    out = torch.zeros(10, 1024, dtype=torch.bfloat16, device="cuda")
    call = lambda **kw: batq.batq_kv_append_mxfp8(  # noqa: E731
        a.cache, kw.pop("tk", a.tk), kw.pop("tv", a.tv), kw.pop("k", k), kw.pop("v", v), kw.pop("slots", slots), positions=kw.pop("pos", pos),
        rope=kw.pop("rope", rope), t_q=kw.pop("tq", a.tq), q=kw.pop("q", q), q_out=kw.pop("q_out", out))
    _refused(batq, NULL, lambda: call(q_out=None))
    _refused(batq, NULL, lambda: call(slots=None))
    _refused(batq, UNSUPPORTED, lambda: call(tq=a.tk))                                   # has a clip
    _refused(batq, UNSUPPORTED, lambda: call(q=None, q_out=None))                        # a query transform and no queries
    _refused(batq, SHAPE, lambda: call(tk=_transforms(batq, 64, 4, 8, 1)[1]))
    _refused(batq, SHAPE, lambda: call(rope=torch.zeros(400, 24, device="cuda")))
    _refused(batq, SHAPE, lambda: call(rope=torch.zeros(400, 256, device="cuda")))
    _refused(batq, SHAPE, lambda: call(rope=rope[:9], pos=None))                         # fewer rows than tokens
    _refused(batq, SHAPE, lambda: call(k=torch.zeros(256, dtype=torch.bfloat16, device="cuda").expand(10, 256)))
    _refused(batq, ALIGN, lambda: call(v=torch.zeros(10, 264, dtype=torch.bfloat16, device="cuda")[:, 4:260]))
    _refused(batq, ALIGN, lambda: call(k=torch.zeros(10, 260, dtype=torch.bfloat16, device="cuda")[:, :256]))
    mid = _transforms(batq, 128, 4, 8, 1)[1]
    batq.batq_transform_set_bf16_intermediates(mid, True)
    _refused(batq, UNSUPPORTED, lambda: call(tk=mid))
    bad = synth.make_transform(128, 3, "paper")
    singular = batq.batq_transform_create(128, bad.left * 0, bad.right)
    _refused(batq, 6, lambda: batq.batq_transform_create_dual(singular))
    torch.cuda.synchronize()
    assert (a.pool[0] == 0x33).all() and (out == 0).all()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("heads,kv_heads,d,page", [(32, 8, 128, 64), (16, 4, 64, 16)])
def test_prompt_then_tokens(batq, heads, kv_heads, d, page):
    """A server's run: two prompts of different length appended and attended over in one call each, then four tokens
    for both, one at a time; every step against attention over the cache as it stands, and against attention over the
    keys and values as they were given, which the transforms leave alone and MXFP8 changes by 2^-4 of each value."""
    g = torch.Generator().manual_seed(77)
    prompts, steps = [50, 83], 4
    pages = 24
    pool = _pool(pages, kv_heads, page, d)
    cache = batq.batq_kv_cache_create(*pool)
    k_t, tk = _transforms(batq, d, 4, 8, 5, clip=False)
    v_t, tv = _transforms(batq, d, 4, 8, 6, clip=False)
    tq = batq.batq_transform_create_dual(tk)
    rope = _table(256, d)
    ids = [torch.randperm(12, generator=g).tolist(), (12 + torch.randperm(12, generator=g)).tolist()]
    table = torch.tensor(ids, dtype=torch.int32).cuda()
    kept = [[], []]        # q, k, v rows of each sequence, rotated, in 64 bits
    lens = [0, 0]
    for step in range(1 + steps):
        rows = prompts if step == 0 else [1, 1]
        x = torch.randn(sum(rows), (heads + 2 * kv_heads) * d, generator=g).bfloat16()
        pos = torch.cat([torch.arange(lens[i], lens[i] + rows[i]) for i in range(2)])
        slots = torch.cat([torch.tensor([ids[i][t // page] * page + t % page for t in range(lens[i], lens[i] + rows[i])]) for i in range(2)])
        q, k, v = x.cuda().split([heads * d, kv_heads * d, kv_heads * d], 1)
        q_out = torch.empty(sum(rows), heads * d, dtype=torch.bfloat16, device="cuda")
        batq.batq_kv_append_mxfp8(cache, tk, tv, k, v, slots.cuda(), positions=pos.int().cuda(), rope=rope.cuda(), t_q=tq, q=q, q_out=q_out)
        lens = [lens[i] + rows[i] for i in range(2)]
        out = torch.empty_like(q_out)
        starts = torch.tensor([0, rows[0], sum(rows)], dtype=torch.int32, device="cuda")
        ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(cache, heads, sum(rows), 2, max(rows), 256))
        batq.batq_attention_kv_mxfp8(cache, q_out, out, torch.tensor(lens, dtype=torch.int32, device="cuda"), table, max(rows), 256, ws, q_starts=starts)
        assert batq.batq_last_device_status() == 0
        kc, ks, vc, vs = (b.cpu() for b in pool)
        used = [ids[i][:-(-lens[i] // page)] for i in range(2)]
        want, _, bound = R.attention(q_out.cpu().unflatten(1, (heads, d)), (kc, ks), (vc, vs), rows, lens, used, d ** -0.5, True)
        got = out.double().cpu().unflatten(1, (heads, d))
        assert ((got - want).abs() <= bound + (want.abs() + bound) * 2.0 ** -8).all()
        # against the unquantised attention: out goes back through P_v^-1
        full = x.double().unflatten(1, (-1, d))
        full[:, :heads + kv_heads] = R.rotate(full[:, :heads + kv_heads], rope[pos])
        pv = torch.linalg.inv(R.dense(v_t.left, v_t.right, d // 32))
        at = 0
        for i in range(2):
            kept[i].append(full[at:at + rows[i]])
            seq = torch.cat(kept[i])
            n, m = lens[i], rows[i]
            qq = seq[n - m:, :heads].transpose(0, 1).unflatten(0, (kv_heads, -1))
            kk, vv = seq[:, heads:heads + kv_heads].transpose(0, 1), seq[:, heads + kv_heads:].transpose(0, 1)
            s = torch.einsum("hgmd,hnd->hgmn", qq, kk) * d ** -0.5
            s = s.masked_fill(torch.arange(n) > torch.arange(m)[:, None] + n - m, -math.inf)
            ref = torch.einsum("hgmn,hnd->hgmd", torch.softmax(s, -1), vv).flatten(0, 1).transpose(0, 1)
            mine = R.transform(got[at:at + m], pv)
            err = float((mine - ref).norm() / ref.norm())
            assert err <= 0.08, err       # E4M3 rounds by at most 2^-4 of a value, 2.6 % in the mean; keys and values both
            at += m
