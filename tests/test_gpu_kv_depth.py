"""The key/value cache's kernels deep inside their loops: rings of tiles refilled many times, slots and barrier phases used
again, several units and items for one CTA, appends with several tiles for one CTA.  Each case asserts that it is that deep."""
import pytest
import torch

import kv_reference as R
from test_gpu_kv_cache import ERR_INDEX, Append

pytestmark = pytest.mark.gpu


class Shared:
    """Many long sequences over one pool: each has the pool's pages in an order of its own.  `bad`: (sequence, page of it)
    whose table entry names no page."""

    def __init__(self, batq, heads, kv_heads, d, page, rows, lens, seed, bad=()):
        g = torch.Generator().manual_seed(seed)
        self.pages_of_pool = -(-max(lens) // page) + 2
        self.k, self.v = [], []
        for dst in (self.k, self.v):
            x = torch.randn(self.pages_of_pool, kv_heads, page, d, generator=g)
            x *= torch.exp(0.5 * torch.randn(self.pages_of_pool, kv_heads, page, 1, generator=g))
            dst.extend(R.mxfp8(x))
        self.cache = batq.batq_kv_cache_create(*[x.cuda() for x in (*self.k, *self.v)])
        counts = [-(-n // page) for n in lens]
        self.pages = [torch.randperm(self.pages_of_pool, generator=g)[:c].tolist() for c in counts]
        table = torch.full((len(lens), max(counts)), 1 << 30, dtype=torch.int32)
        for i, p in enumerate(self.pages):
            table[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
        self.hidden = [None] * len(lens)
        for i, at in bad:
            table[i, at] = -1 if at % 2 else self.pages_of_pool
            h = torch.zeros(lens[i], dtype=torch.bool) if self.hidden[i] is None else self.hidden[i]
            h[at * page:(at + 1) * page] = True
            self.hidden[i] = h
        self.table, self.status = table.cuda(), ERR_INDEX if bad else 0
        self.rows, self.lens, self.heads, self.kv_heads, self.d = rows, lens, heads, kv_heads, d
        self.q = (2 * torch.randn(sum(rows), heads, d, generator=g)).bfloat16()
        self.starts = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32)

    def run(self, batq):
        q = self.q.cuda().flatten(1)
        out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0], self.heads), 5.0, device="cuda")
        sizes = (self.heads, q.shape[0], len(self.lens), max(self.rows), max(self.lens))
        ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(self.cache, *sizes))
        ws.fill_(0xFF)
        batq.batq_attention_kv_mxfp8(self.cache, q, out, torch.tensor(self.lens, dtype=torch.int32).cuda(), self.table, *sizes[3:], ws,
                                     q_starts=self.starts.cuda(), lse=lse)
        assert batq.batq_last_device_status() == self.status
        return out.unflatten(1, (self.heads, self.d)).double().cpu(), lse.double().cpu()

    def check(self, out, lse, picks):
        """Rows `picks`, (sequence, row of it), against 64 bits: each as a sequence of one row that ends with the last key it sees."""
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        at = [int(self.starts[i]) + j for i, j in picks]
        lens = [self.lens[i] - self.rows[i] + j + 1 for i, j in picks]
        hidden = [torch.zeros(n, dtype=torch.bool) if self.hidden[i] is None else self.hidden[i] for (i, _), n in zip(picks, lens)]
        scale = self.d ** -0.5
        want, wlse, bound = R.attention(self.q[at], self.k, self.v, [1] * len(picks), lens, [self.pages[i] for i, _ in picks], scale, True, hidden)
        limit = bound + (want.abs() + bound) * 2.0 ** -8
        far = (out[at] - want).abs() / limit
        assert far.max() <= 1, f"{int((far > 1).sum())} of {far.numel()} too far, worst {float(far.max()):.2f} of the bound"
        big = float(R.values(*self.k).norm(dim=-1).max() * self.q.double().norm(dim=-1).max()) * scale
        assert ((lse[at] - wlse).abs() <= 2.0 ** -16 + wlse.abs() * 2.0 ** -22 + big * (self.d + 8) * 2.0 ** -24).all()


@pytest.mark.parametrize("heads,kv_heads,d,page,rows,unit", [(32, 8, 128, 64, 1, 8), (32, 8, 128, 16, 3, 16), (28, 4, 128, 32, 3, 24),
                                                             (4, 4, 64, 128, 1, 8), (16, 4, 64, 64, 4, 16), (16, 4, 64, 16, 5, 24)])
def test_decode_deep(batq, heads, kv_heads, d, page, rows, unit):
    """More than 128 tiles of one unit for a CTA, so more than 32 for each of its warps: 16 turns of the ring, a second
    look-up of pages.  Units of 8, 16 and 24 rows; pages missing at the beginning and late in a sequence."""
    g = torch.Generator().manual_seed(unit + d)
    n_rows, ctas = rows * heads // kv_heads, (3 if unit == 8 else 2) * torch.cuda.get_device_properties(0).multi_processor_count
    assert unit - 8 < n_rows <= unit and (unit != 24 or n_rows > 16)
    seqs = -(-150 * ctas // (kv_heads * 140))
    lens = torch.randint(4500, 5000, (seqs,), generator=g).tolist()
    cost = sum(kv_heads * (-(-n // 32) + 12) for n in lens)      # of all units, in tiles
    assert cost // ctas - 12 > 128 and lens[0] > 32 * 140        # the first CTA's share of the first unit
    b = Shared(batq, heads, kv_heads, d, page, [rows] * seqs, lens, 31 + unit, bad=((0, 2), (0, 5), (1, 3), (2, lens[2] // page - 1)))
    out, lse = b.run(batq)
    picks = [(i, rows - 1 - i % rows) for i in (0, 1, 2, 3, seqs // 2, seqs - 1)]
    b.check(out, lse, picks)


@pytest.fixture(params=[1, 2], ids=["codes", "copy"])
def copy_path(batq, request):
    batq.batq_debug_force_attention_copy(request.param)
    yield request.param
    batq.batq_debug_force_attention_copy(0)


@pytest.mark.parametrize("heads,kv_heads,d,page,rows,lens", [(32, 8, 128, 64, [1300, 1250], [1700, 1300]), (16, 4, 64, 16, [2600, 2500], [3300, 2500])])
def test_prompts_deep(batq, heads, kv_heads, d, page, rows, lens, copy_path):
    """Three items for some CTAs and two for the others, of up to 14 or 26 tiles: scale slots, stages and barriers used again
    within an item and across items, whose last M tile is empty for some; pages missing in the second sequence."""
    ctas = torch.cuda.get_device_properties(0).multi_processor_count
    units = sum(kv_heads * -(-m * (heads // kv_heads) // 256) for m in rows)
    assert units > 2 * ctas and min(lens) > 8 * 128 and any(0 < m * (heads // kv_heads) % 256 <= 128 for m in rows)
    b = Shared(batq, heads, kv_heads, d, page, rows, lens, 41, bad=((1, 1), (1, lens[1] // page - 2)))
    # a row of the second sequence that sees none but missing pages' keys would be empty: page 0 is there
    out, lse = b.run(batq)
    picks = [(i, j) for i in (0, 1) for j in (0, 1, 63, 64, 200, rows[i] // 2, rows[i] - 130, rows[i] - 20, rows[i] - 1)]
    b.check(out, lse, picks)


@pytest.mark.parametrize("rows,lens", [([70], [40000]), ([65, 65], [9001, 20011])])
def test_chunk_far_behind(batq, rows, lens, copy_path):
    """A chunk of a prompt far into a document: each unit in several parts, of more than 8 tiles."""
    kv_heads, ctas = 8, torch.cuda.get_device_properties(0).multi_processor_count
    units = sum(kv_heads * -(-m * 4 // 256) for m in rows)
    assert -(-max(lens) // 128) // (2 * ctas // units) > 8
    b = Shared(batq, 32, kv_heads, 128, 128, rows, lens, 51)
    out, lse = b.run(batq)
    b.check(out, lse, [(i, j) for i in range(len(rows)) for j in (0, rows[i] - 1)])


@pytest.mark.parametrize("heads,kv_heads,d", [(28, 4, 128), (32, 8, 64), (5, 3, 128), (40, 7, 64)])
@pytest.mark.parametrize("gr,gc", [(4, 8), (8, 4)])
def test_append_deep(batq, heads, kv_heads, d, gr, gc):
    """Several tiles of each role for a CTA: both stages, the fetch ahead, the steps from tile to tile."""
    per_tile, ctas = 256 // (d // 32), 3 * torch.cuda.get_device_properties(0).multi_processor_count
    tokens = -(-4 * ctas * per_tile // (heads + 2 * kv_heads)) + 37
    assert tokens * (heads + 2 * kv_heads) > 4 * ctas * per_tile
    a = Append(batq, tokens, heads, kv_heads, d, 32, rot=d, gr=gr, gc=gc, seed=21, padding=(3, tokens // 2, tokens - 1))
    a.run(batq)
    assert batq.batq_last_device_status() == 0
    a.check()


def test_rows_of_sound_sequences_beside_nonsense(batq):
    """Row starts of which some run backwards or past the end: the sequences whose own starts are in order come out right."""
    heads, lens = 8, [40, 50, 60]
    b = Shared(batq, heads, 2, 128, 32, [2, 3, 2], lens, 61)
    q = b.q.cuda().flatten(1)
    for starts, seq in (([0, 2, 1 << 30, 7], 0), ([1 << 30, -(1 << 31), 5, 7], 2)):
        out, lse = torch.full_like(q, 7.0), torch.full((7, heads), 5.0, device="cuda")
        ws = batq.aligned_workspace(batq.batq_attention_kv_mxfp8_workspace_bytes(b.cache, heads, 7, 3, 3, 60))
        batq.batq_attention_kv_mxfp8(b.cache, q, out, torch.tensor(lens, dtype=torch.int32).cuda(), b.table, 3, 60, ws,
                                     q_starts=torch.tensor(starts, dtype=torch.int32).cuda(), lse=lse)
        assert batq.batq_last_device_status() == 0
        at = int(b.starts[seq])
        want, _, bound = R.attention(b.q[at:at + 2], b.k, b.v, [2], [lens[seq]], [b.pages[seq]], 128 ** -0.5, True)
        got = out[at:at + 2].unflatten(1, (heads, 128)).double().cpu()
        assert ((got - want).abs() <= bound + (want.abs() + bound) * 2.0 ** -8).all()
