// Attention over the paged MXFP8 key/value cache for a few query rows per key/value head (decoding, drafts).
//
//   o = sum_t softmax_t(scale * q . k_t) v_t,   k_t = 2^ek[t,b] kc[t], v_t = 2^ev[t,b] vc[t]   (b: 32-channel block)
//
// Bound by the cache's bytes: 33/32 * 2 * head_dim per token and head, read once.  Query rows of one sequence and one
// key/value head (rows = query rows x heads of the group) share every byte: up to 8 * NT of them are one unit.  The
// tiles (32 tokens) of all units of the batch stand in one line, cut into ranges of equal cost, one for each CTA that the device
// holds at once: a ragged batch, one long sequence and many short ones all keep every SM at work to the end.  (A CTA per
// fixed piece of a sequence instead: 33 against 25 us for 16 sequences of up to 4001 keys, 137 against 58 for one of
// 131072, 124 against 110 for 128 of up to 8192.)  A cut never falls into a unit of up to kAtSnap tiles; what a cut
// divides is joined from the workspace, in the order of the tokens, by attention_join_kernel.
//
// Within a range a CTA's four warps take every fourth tile and are independent of one another until the unit ends: each
// has a ring of tiles filled by TMA, a running maximum and sum, and an accumulator; they meet in shared memory.
//
// The products run on f16 matrix instructions (m16n8k16, fp32 sums), tokens or channels as the 16 rows and query rows as
// the 8 columns, because eight query rows would leave half of a 128-row tensor-memory tile's lanes and more unused while
// the codes would still have to be widened.  E4M3 is exact in f16; the scales are kept apart from it:
//   scores   S = sum_b 2^ek[t,b] (q_b . kc_b): one fp32 factor per token and block on the accumulators.  q is scaled by
//            a power of two per row so that its largest element is in [2^14, 2^15): exact in f16 down to 2^-31 of it.
//   values   vc 2^(ev - c) in f16 with c one integer per token (its largest ev, less 7): exact within 2^22 of the token's
//            largest block.  c joins the exponent of the softmax weight, w = 2^(s + c - m) with m the reference, 2^7 below
//            the row's largest s + c when it was set.  So w, in f16, is off by 2^-11 of itself or by 2^-32 of the row's
//            largest *contribution* to the output, not of its largest probability: a token of large probability and tiny
//            values (an attention sink) leaves the others their bits.  The softmax sum takes 2^-c w in fp32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_append.cuh"
#include "ptx.cuh"

namespace batq {

constexpr int kAtWarps = 4;
constexpr int kAtTile = 32;       // tokens a warp takes at a time
constexpr int kAtStages = 2;       // x 8.4 KB x 4 warps: three CTAs on an SM
constexpr int kAtSnap = 8;        // units of up to this many tiles are not divided
constexpr int kAtMaxSeqs = 512;   // sequences of one launch
constexpr int kAtUnitCost = 12;   // what a unit costs besides its tiles, in tiles (look-ups, first loads, the merge; 6: 115 us, 8: 113, 12: 110 for 128 ragged sequences)
constexpr float kAtHead = 7.0f;   // log2 of a row's largest weight when its reference is set: f16 has no bits below 2^-24
constexpr float kAtMost = 15.0f;  // log2 of the largest weight that leaves the reference where it is: f16 ends at 2^16
constexpr float kAtNone = -1e30f; // the reference of a row that has seen no key
// Least c: 2^-c times a weight is a term of the softmax sum in fp32, of tokens without any value too.
constexpr int kAtMinScale = -64;

struct AttnJoin {
  int32_t parts;     // CTAs that share the unit, this one among them; 0: none starts here
  int32_t row0, n_rows, head;
  int64_t q0;        // the sequence's first query row
};

struct AttnParams {
  const uint16_t* q;          // bf16 bits, row (token, head) at token * ldq + head * head_dim
  int64_t ldq;
  int32_t q_heads, kv_heads, group;
  int64_t tokens;             // rows of q
  const int32_t* q_starts;    // [seqs + 1] or NULL: row i is sequence i
  const int32_t* kv_lens;     // [seqs]
  const int32_t* page_table;  // [seqs][ld_pages]
  int64_t ld_pages;
  int32_t max_q, max_kv;
  int32_t page_shift;
  int32_t pages;
  const uint8_t* k_scales;
  const uint8_t* v_scales;
  float scale_log2;           // scale * log2(e)
  int32_t causal;
  uint16_t* out;              // bf16, row (token, head) at token * ldo + head * head_dim
  int64_t ldo;
  float* lse;                 // [tokens][q_heads] or NULL
  int32_t seqs;               // of this launch, at most kAtMaxSeqs
  int32_t most_rows;          // sequences with more rows (query rows x group) are another kernel's
  int32_t seq0;               // row of its first sequence where q_starts is NULL
  float* part_o;              // [CTA][2][rows][head_dim]: sums relative to part_ml's reference
  float2* part_ml;            // [CTA][2][rows]: reference m, softmax sum
  AttnJoin* join;             // [CTA]: the unit that starts in its range and ends in another's
};

template <int D, int NT>
struct AttnCfg {
  static constexpr int kRows = 8 * NT;
  static constexpr int kBlocks = D / 32;
  static constexpr int kCodeBytes = kAtTile * D;                   // of K or V
  static constexpr int kStageBytes = 2 * kCodeBytes;
  static constexpr int kScaleBytes = kAtTile * kBlocks;            // of K or V
  static constexpr int kRing = kAtWarps * kAtStages * kStageBytes;
  static constexpr int kScales = kAtWarps * kAtStages * 2 * kScaleBytes;
  static constexpr int kMult = kAtWarps * kBlocks * kAtTile * 2;   // 2^(ev - c) of the tokens of a warp's tile, f16
  static constexpr int kKeyMult = kAtWarps * kBlocks * kAtTile * 4; // 2^ek, fp32
  static constexpr int kSmemBytes = kRing + kScales + kMult + kKeyMult + 1024;
  static constexpr int kCtasPerSm = NT == 1 ? 3 : 2;   // by shared memory; by registers
  static_assert(kAtWarps * kRows * (D + 2) * 4 <= kRing, "the merge of the warps goes through the ring");
};

// What one sequence of the batch asks for, cut to what the call's arguments allow.
struct AttnSeq {
  int64_t q0;    // first query row
  int32_t nq, len;
};
__device__ __forceinline__ AttnSeq attn_seq(const AttnParams& p, int seq) {
  AttnSeq s;
  if (p.q_starts == nullptr) {
    s.q0 = p.seq0 + seq;
    s.nq = 1;
  } else {
    const int64_t a = p.q_starts[seq], b = p.q_starts[seq + 1];
    s.q0 = min(max(a, int64_t(0)), p.tokens);
    s.nq = static_cast<int32_t>(min(max(min(b, p.tokens) - s.q0, int64_t(0)), static_cast<int64_t>(p.max_q)));
  }
  const int64_t room = p.ld_pages << p.page_shift;
  s.len = static_cast<int32_t>(max(int64_t(0), min(min(static_cast<int64_t>(p.kv_lens[seq]), static_cast<int64_t>(p.max_kv)), room)));
  return s;
}
// Keys that query row qi of a sequence sees: the first `return` ones.
__device__ __forceinline__ int attn_visible(const AttnParams& p, const AttnSeq& s, int qi) {
  return p.causal ? max(0, min(s.len, s.len - s.nq + qi + 1)) : s.len;
}

__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w) {   // the low 16 bits
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2_high(uint32_t w) {   // the high 16 bits
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same into fresh accumulators.
__device__ __forceinline__ void mma_16816_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ float ex2(float x) {   // results below 2^-126 are 0: nothing here tells them from it
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float pow2i(int e) {   // 2^e, e in [-126, 127]
  return __int_as_float((e + 127) << 23);
}
__device__ __forceinline__ uint32_t largest_byte(uint32_t w) {
  const uint32_t top = __vmaxu4(w, w >> 16);
  return max(top & 255u, (top >> 8) & 255u);
}
// 2^e as f16 bits; 0 below 2^-24 (e <= 7 here).
__device__ __forceinline__ uint32_t f16_pow2(int e) {
  return e >= -14 ? static_cast<uint32_t>(e + 15) << 10 : e >= -24 ? 1u << (e + 24) : 0u;
}
// The same of two scale bytes in the halves of a word, less d (the whole warp calls it).
__device__ __forceinline__ uint32_t f16_pow2x2(uint32_t bytes, int d) {
  const uint32_t e = __vmaxs2(__vsub2(bytes, (d - 15) * 0x10001u), 0u);
  if (__any_sync(0xFFFFFFFFu, (e & 0xFFFFu) == 0u || e < 0x10000u))   // a factor below 2^-14: subnormal f16
    return f16_pow2(static_cast<int>(bytes & 0xFFFFu) - d) | f16_pow2(static_cast<int>(bytes >> 16) - d) << 16;
  return e << 10;
}

// The token of a tile's eight-token group that stands in row i of a matrix fragment.  Rows 0..3 are read by the first
// half of the warp: with these, eight-byte reads of the swizzled rows meet all banks once.
template <int D>
__device__ __forceinline__ int frag_token(int i) {
  return D == 128 ? ((i & 3) << 1) | (i >> 2) : ((i & 2) << 1) | ((i >> 2) << 1) | (i & 1);
}
template <int D>
__device__ __forceinline__ int token_frag(int t) {   // its inverse
  return D == 128 ? ((t & 1) << 2) | (t >> 1) : ((t & 2) << 1) | ((t >> 2) << 1) | (t & 1);
}
// Byte offset of 16-byte chunk `c` of row `row` in a tile as TMA's 128-byte (D = 128) or 64-byte swizzle leaves it.
template <int D>
__device__ __forceinline__ uint32_t tile_offset(int row, int c) {
  return D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}

__device__ __forceinline__ void store_attn_row(const AttnParams& p, int64_t token, int head, int D, int ch, float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  *reinterpret_cast<__nv_bfloat162*>(p.out + token * p.ldo + static_cast<int64_t>(head) * D + ch) = v;
}

// Tiles of a unit of a sequence with `len` keys (one at least: its rows are written all the same), and its units: the
// key/value heads times the row tiles.  A row tile counts all of the sequence's tiles, those that its rows do not see too.
__device__ __forceinline__ int attn_tiles(int len) { return max(1, (len + kAtTile - 1) / kAtTile); }
template <int NT>
__device__ __forceinline__ int attn_units(const AttnParams& p, const AttnSeq& s) {
  const int rows = s.nq * p.group;
  return rows > p.most_rows ? 0 : p.kv_heads * ((rows + 8 * NT - 1) / (8 * NT));
}

template <int D, int NT>
__global__ void __launch_bounds__(kAtWarps * 32, AttnCfg<D, NT>::kCtasPerSm)
attention_kv_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ AttnParams p) {
  using Cfg = AttnCfg<D, NT>;
  constexpr int BL = Cfg::kBlocks;
  extern __shared__ __align__(1024) uint8_t at_smem[];
  __shared__ __align__(8) uint64_t bars[kAtWarps * kAtStages];
  __shared__ int first[kAtMaxSeqs];        // the cost of all units in front of each sequence's
  __shared__ int weight[kAtMaxSeqs];       // the cost of one of its units: its tiles + kAtUnitCost
  __shared__ int warp_sum[kAtWarps];
  __shared__ int2 warp_count[kAtWarps];
  __shared__ int abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(at_smem) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = base + warp * (kAtStages * Cfg::kStageBytes);
  uint8_t* scales = base + Cfg::kRing + warp * (kAtStages * 2 * Cfg::kScaleBytes);
  uint16_t* mult = reinterpret_cast<uint16_t*>(base + Cfg::kRing + Cfg::kScales) + warp * (BL * kAtTile);
  float* kmult = reinterpret_cast<float*>(base + Cfg::kRing + Cfg::kScales + Cfg::kMult) + warp * (BL * kAtTile);

  grid_launch_dependents();
  if (lane == 0) {
    for (int i = 0; i < kAtStages; ++i) mbar_init(smem_u32(&bars[warp * kAtStages + i]), 1);
    mbar_fence_init();
  }
  if (tid == 0) {
    abort_flag = 0;
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  grid_dependency_wait();   // q, the lengths and the cache may come from the grid in front

  // the cost in front of each sequence, and of all; this CTA's range and the sequence that it starts in
  int pos, stop, seq, chunk;
  {
    const int per = (p.seqs + kAtWarps * 32 - 1) / (kAtWarps * 32);
    const int s0 = min(p.seqs, tid * per), s1 = min(p.seqs, s0 + per);
    int sum = 0;
    for (int s = s0; s < s1; ++s) {
      first[s] = sum;
      const AttnSeq q = attn_seq(p, s);
      weight[s] = attn_tiles(q.len) + kAtUnitCost;
      sum += attn_units<NT>(p, q) * weight[s];
    }
    int scan = sum;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, scan, x);
      if (lane >= x) scan += v;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    int before = scan - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kAtWarps; ++w) {
      if (w < warp) before += warp_sum[w];
      total += warp_sum[w];
    }
    chunk = max(kAtWarps, static_cast<int>((static_cast<uint32_t>(total) + gridDim.x - 1) / gridDim.x));
    const int64_t x0 = static_cast<int64_t>(chunk) * blockIdx.x, x1 = x0 + chunk;
    int2 n = make_int2(0, 0);   // sequences that start at or before x0, x1
    for (int s = s0; s < s1; ++s) {
      const int f = first[s] + before;
      first[s] = f;
      n.x += f <= x0;
      n.y += f <= x1;
    }
    n.x = __reduce_add_sync(0xFFFFFFFFu, n.x);
    n.y = __reduce_add_sync(0xFFFFFFFFu, n.y);
    if (lane == 0) warp_count[warp] = n;
    __syncthreads();
    n = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < kAtWarps; ++w) {
      n.x += warp_count[w].x;
      n.y += warp_count[w].y;
    }
    // A cut stays where it is in a long unit behind what the unit costs before its first tile, else it goes back to the
    // start of the unit.  (The last sequence that starts at or before it has rows: those without start where the next does.)
    auto cut = [&](int64_t x, int s) {
      if (x >= total) return total;
      const int w = weight[s], in = (static_cast<int>(x) - first[s]) % w;
      return static_cast<int>(x) - (w <= kAtSnap + kAtUnitCost || in <= kAtUnitCost ? in : 0);
    };
    seq = n.x - 1;
    pos = cut(x0, n.x - 1);
    stop = cut(x1, n.y - 1);
  }
  AttnJoin join{};
  bool ok = true;
  int turn = 0;             // tiles this warp has taken, over all units

  while (pos < stop) {
    AttnSeq sq = attn_seq(p, seq);
    while (pos >= first[seq] + attn_units<NT>(p, sq) * weight[seq]) sq = attn_seq(p, ++seq);   // the next one with rows
    const int unit = (pos - first[seq]) / weight[seq], unit_tiles = weight[seq] - kAtUnitCost;
    const int unit0 = first[seq] + unit * weight[seq] + kAtUnitCost;   // its first tile
    const int tile0 = max(0, pos - unit0), tile1 = min(unit_tiles, stop - unit0);
    pos = unit0 + tile1;
    const int head = unit % p.kv_heads, row0 = unit / p.kv_heads * Cfg::kRows;
    const int n_rows = min(Cfg::kRows, sq.nq * p.group - row0);
    const int end = attn_visible(p, sq, (row0 + n_rows - 1) / p.group);   // keys the last row sees

    if (end <= 0 && unit_tiles == 1) {   // nothing to see, nothing to join
      for (int i = tid; i < n_rows * (D / 2); i += kAtWarps * 32) {
        const int row = row0 + i / (D / 2), ch = i % (D / 2) * 2;
        const int64_t token = sq.q0 + row / p.group;
        const int qh = head * p.group + row % p.group;
        store_attn_row(p, token, qh, D, ch, 0.0f, 0.0f);
        if (ch == 0 && p.lse != nullptr) p.lse[token * p.q_heads + qh] = -INFINITY;
      }
      continue;
    }

    // this warp's tiles: tile0 + warp + 4 i, i < n
    const int last = min(tile1, (end + kAtTile - 1) / kAtTile);
    const int n = ok && last - tile0 > warp ? (last - tile0 - warp + kAtWarps - 1) / kAtWarps : 0;
    const int32_t* pages = p.page_table + static_cast<int64_t>(seq) * p.ld_pages;
    const int parts = p.page_shift == 4 ? 2 : 1;   // pages of a tile
    // The pages of the next 32 tiles to load, one per lane (two for 16-token pages): the look-up is off the tiles' path.
    int page_a = 0, page_b = 0;
    auto look_up = [&](int i) {
      page_a = page_b = -1;
      if (i + lane < n) {
        const int tok = (tile0 + warp + kAtWarps * (i + lane)) * kAtTile;
        page_a = pages[tok >> p.page_shift];
        if (parts == 2 && tok + 16 < end) page_b = pages[(tok >> 4) + 1];
      }
    };
    // One page's part of a tile: `rows` tokens from token `off` of the page, to row `at` of stage st.
    auto load = [&](int st, int page, int off, int rows, int at) {
      const int row = ((page * p.kv_heads + head) << p.page_shift) + off;   // below 2^31
      const uint32_t bar = smem_u32(&bars[warp * kAtStages + st]);
      const uint32_t dst = smem_u32(ring + st * Cfg::kStageBytes) + at * D;
      const uint32_t sdst = smem_u32(scales + st * 2 * Cfg::kScaleBytes) + at * BL;
      const int64_t soff = static_cast<int64_t>(row) * BL;
      tma_load_2d(dst, &tmap_k, 0, row, bar);
      bulk_g2s(sdst, p.k_scales + soff, rows * BL, bar);
      tma_load_2d(dst + Cfg::kCodeBytes, &tmap_v, 0, row, bar);
      bulk_g2s(sdst + Cfg::kScaleBytes, p.v_scales + soff, rows * BL, bar);
    };
    uint32_t bad = 0;   // bits 2 s, 2 s + 1: the first / second part of the tile in stage s is not there
    auto issue = [&](int i) {
      if ((i & 31) == 0) look_up(i);
      const int st = (turn + i) % kAtStages;
      const int tok = (tile0 + warp + kAtWarps * i) * kAtTile;
      const uint32_t bar = smem_u32(&bars[warp * kAtStages + st]);
      const int pa = __shfl_sync(0xFFFFFFFFu, page_a, i & 31);
      const bool lost = static_cast<uint32_t>(pa) >= static_cast<uint32_t>(p.pages);
      uint32_t miss = lost ? 1u : 0u;
      if (parts == 1) {
        if (lane == 0) {
          mbar_arrive_expect_tx(bar, lost ? 0 : kAtTile * 2 * (D + BL));
          if (!lost) load(st, pa, tok & ((1 << p.page_shift) - 1), kAtTile, 0);
        }
      } else {
        const int pb = __shfl_sync(0xFFFFFFFFu, page_b, i & 31);
        const bool second = tok + 16 < end, lost_b = second && static_cast<uint32_t>(pb) >= static_cast<uint32_t>(p.pages);
        miss |= lost_b ? 2u : 0u;
        if (lane == 0) {
          mbar_arrive_expect_tx(bar, ((lost ? 0 : 1) + (second && !lost_b ? 1 : 0)) * 16 * 2 * (D + BL));
          if (!lost) load(st, pa, 0, 16, 0);
          if (second && !lost_b) load(st, pb, 0, 16, 16);
        }
      }
      if (miss != 0 && lane == 0) atomicOr(&g_device_error, kErrorIndex);
      bad = (bad & ~(3u << (2 * st))) | (miss << (2 * st));
    };
    int issued = 0;
    for (; issued < kAtStages && issued < n; ++issued) issue(issued);

    // q as the matrix instruction's B fragments, scaled by a power of two per row
    uint32_t qf[NT][BL][4];
    float qs[NT][2];      // the factor of rows 2 t4, 2 t4 + 1 on the accumulators
    int lim[NT][2];       // keys those rows see
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int row = row0 + j * 8 + g;
      float v[BL][8];
      float amax = 0.0f;
#pragma unroll
      for (int b = 0; b < BL; ++b) {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (j * 8 + g < n_rows)
          w = ld_global_ordered_v4(p.q + (sq.q0 + row / p.group) * p.ldq + static_cast<int64_t>(head * p.group + row % p.group) * D + b * 32 + t4 * 8);
        unpack_bf16x8(w, v[b]);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[b][i]));
      }
      amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
      const int e = max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -100);
      const float up = pow2i(14 - e);
#pragma unroll
      for (int b = 0; b < BL; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __half2 h = __floats2half2_rn(v[b][2 * i] * up, v[b][2 * i + 1] * up);
          qf[j][b][i] = *reinterpret_cast<const uint32_t*>(&h);
        }
      const float f = p.scale_log2 * pow2i(e - 14);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        qs[j][i] = __shfl_sync(0xFFFFFFFFu, f, (2 * t4 + i) * 4);
        const int rr = j * 8 + 2 * t4 + i;
        lim[j][i] = rr < n_rows ? attn_visible(p, sq, (row0 + rr) / p.group) : 0;
      }
    }
    const int full = attn_visible(p, sq, row0 / p.group);   // keys that every row sees

    float o[D / 16][NT][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      m[j][0] = m[j][1] = kAtNone;
      l[j][0] = l[j][1] = 0.0f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[c][j][i] = 0.0f;
    }

    const uint32_t mult_addr = smem_u32(mult);
    for (int i = 0; i < n; ++i) {
      const int st = (turn + i) % kAtStages;
      const uint32_t bar = smem_u32(&bars[warp * kAtStages + st]);
      ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(bar, ((turn + i) / kAtStages) & 1, &abort_flag));
      if (!ok) break;
      const int tok0 = (tile0 + warp + kAtWarps * i) * kAtTile;
      const uint32_t kt = smem_u32(ring + st * Cfg::kStageBytes), vt = kt + Cfg::kCodeBytes;
      const uint8_t* ks = scales + st * 2 * Cfg::kScaleBytes;
      const uint8_t* vs = ks + Cfg::kScaleBytes;
      const uint32_t miss = (bad >> (2 * st)) & 3u;
      const bool whole = tok0 + kAtTile <= full && miss == 0;   // every row sees every token
      const bool here = tok0 + lane < end && !((miss >> (parts == 2 ? lane >> 4 : 0)) & 1u);   // the lane's token
      if (tok0 + kAtTile > end || miss != 0) {
        // what stands behind the last token (or on a page that is not there) may be anything, NaN codes too
        if (!here) {
#pragma unroll
          for (int c = 0; c < D / 16; ++c)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vt + lane * D + c * 16), "r"(0u) : "memory");
        }
      }
      // the value scales of the lane's token, their common exponent, and the f16 factors 2^(ev - c)
      int c_lane;
      {
        uint32_t w;
        if (BL == 4) w = *reinterpret_cast<const uint32_t*>(vs + lane * 4);
        else w = *reinterpret_cast<const uint16_t*>(vs + lane * 2);
        uint32_t kw;
        if (BL == 4) kw = *reinterpret_cast<const uint32_t*>(ks + lane * 4);
        else kw = *reinterpret_cast<const uint16_t*>(ks + lane * 2);
        uint32_t kf[BL];
#pragma unroll
        for (int b = 0; b < BL; ++b) kf[b] = __byte_perm(kw, 0u, 0x0444 | b << 12) >> 1;   // the byte to the exponent field
        if (BL == 4) *reinterpret_cast<uint4*>(kmult + lane * 4) = make_uint4(kf[0], kf[1], kf[BL - 2], kf[BL - 1]);
        else *reinterpret_cast<uint2*>(kmult + lane * 2) = make_uint2(kf[0], kf[1]);
        if (!here) w = 0;
        c_lane = max(static_cast<int>(largest_byte(w)) - 127 - 7, kAtMinScale);
        const int at = (lane & 24) | token_frag<D>(lane & 7);
#pragma unroll
        for (int b = 0; b < BL; b += 2) {   // two blocks in the halves of a word
          const uint32_t f = f16_pow2x2(__byte_perm(w, 0u, b == 0 ? 0x4140 : 0x4342), c_lane + 127);
          mult[b * kAtTile + at] = static_cast<uint16_t>(f);
          mult[(b + 1) * kAtTile + at] = static_cast<uint16_t>(f >> 16);
        }
      }
      __syncwarp();

      // S^T [32 tokens x rows] in log2 units, plus c
      float s[2][NT][4];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const int ta = mt * 16 + frag_token<D>(g), tb = ta + 8;
        float fa[BL], fb[BL];
        if (BL == 4) {
          *reinterpret_cast<float4*>(fa) = *reinterpret_cast<const float4*>(kmult + ta * 4);
          *reinterpret_cast<float4*>(fb) = *reinterpret_cast<const float4*>(kmult + tb * 4);
        } else {
          *reinterpret_cast<float2*>(fa) = *reinterpret_cast<const float2*>(kmult + ta * 2);
          *reinterpret_cast<float2*>(fb) = *reinterpret_cast<const float2*>(kmult + tb * 2);
        }
#pragma unroll
        for (int b = 0; b < BL; ++b) {
          uint32_t a0, a1, b0, b1;
          asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(a0), "=r"(a1) : "r"(kt + tile_offset<D>(ta, 2 * b + (t4 >> 1)) + (t4 & 1) * 8) : "memory");
          asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(b0), "=r"(b1) : "r"(kt + tile_offset<D>(tb, 2 * b + (t4 >> 1)) + (t4 & 1) * 8) : "memory");
          const uint32_t f0[4] = {e4m3x2_to_f16x2(a0), e4m3x2_to_f16x2(b0), e4m3x2_to_f16x2_high(a0), e4m3x2_to_f16x2_high(b0)};
          const uint32_t f1[4] = {e4m3x2_to_f16x2(a1), e4m3x2_to_f16x2(b1), e4m3x2_to_f16x2_high(a1), e4m3x2_to_f16x2_high(b1)};
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            float d[4];
            mma_16816_first(d, f0, qf[j][b][0], qf[j][b][1]);
            mma_16816(d, f1, qf[j][b][2], qf[j][b][3]);
            s[mt][j][0] = b == 0 ? d[0] * fa[b] : fmaf(d[0], fa[b], s[mt][j][0]);
            s[mt][j][1] = b == 0 ? d[1] * fa[b] : fmaf(d[1], fa[b], s[mt][j][1]);
            s[mt][j][2] = b == 0 ? d[2] * fb[b] : fmaf(d[2], fb[b], s[mt][j][2]);
            s[mt][j][3] = b == 0 ? d[3] * fb[b] : fmaf(d[3], fb[b], s[mt][j][3]);
          }
        }
      }
      // Weights against the reference m: it follows the maximum only where that has grown by more than 2^8, so that
      // most tiles exchange nothing between the lanes and leave the accumulators alone.
      float cf[2][2], unscale[2][2];   // c, 2^-c of the thread's four tokens
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = __shfl_sync(0xFFFFFFFFu, c_lane, mt * 16 + h * 8 + frag_token<D>(g));
          cf[mt][h] = static_cast<float>(c);
          unscale[mt][h] = pow2i(-c);
        }
      float z[2][NT][4];
      auto weigh = [&] {   // exponents of the weights; returns the largest
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) z[mt][j][x] = fmaf(s[mt][j][x], qs[j][x & 1], cf[mt][x >> 1] - m[j][x & 1]);
        if (!whole) {
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int tt = mt * 16 + (x >> 1) * 8 + frag_token<D>(g);
                if (tok0 + tt >= lim[j][x & 1] || ((miss >> (parts == 2 ? tt >> 4 : 0)) & 1u)) z[mt][j][x] = -INFINITY;
              }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) top = fmaxf(top, fmaxf(z[0][j][x], z[1][j][x]));
        return top;
      };
      if (__any_sync(0xFFFFFFFFu, weigh() > kAtMost)) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float top = kAtNone;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (z[mt][j][x + 2 * h] > -INFINITY) top = fmaxf(top, fmaf(s[mt][j][x + 2 * h], qs[j][x], cf[mt][h]));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
            const float mn = fmaxf(m[j][x], top - kAtHead), alpha = ex2(m[j][x] - mn);
            m[j][x] = mn;
            l[j][x] *= alpha;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
              o[c][j][x] *= alpha;
              o[c][j][x + 2] *= alpha;
            }
          }
        weigh();
      }
      uint32_t pf[2][NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float sum = 0.0f;
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            z[mt][j][x] = ex2(z[mt][j][x]);
            z[mt][j][x + 2] = ex2(z[mt][j][x + 2]);
            sum = fmaf(z[mt][j][x], unscale[mt][0], sum);
            sum = fmaf(z[mt][j][x + 2], unscale[mt][1], sum);
          }
          l[j][x] += sum;
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const __half2 w = __floats2half2_rn(z[mt][j][2 * h], z[mt][j][2 * h + 1]);
            pf[mt][j][h] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&w));
          }
      }
      // O^T += V^T P^T
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        const int row = mt * 16 + ((lane >> 3) & 1) * 8 + frag_token<D>(lane & 7);
#pragma unroll
        for (int b = 0; b < BL; ++b) {
          uint32_t w[4], s0, s1;
          ldmatrix_x4_trans(w, vt + tile_offset<D>(row, 2 * b + (lane >> 4)));
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(s0) : "r"(mult_addr + (b * kAtTile + mt * 16 + 2 * t4) * 2) : "memory");
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(s1) : "r"(mult_addr + (b * kAtTile + mt * 16 + 8 + 2 * t4) * 2) : "memory");
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t u0 = __byte_perm(w[2 * c], 0u, 0x3120), u1 = __byte_perm(w[2 * c + 1], 0u, 0x3120);
            const uint32_t f[4] = {hmul2(e4m3x2_to_f16x2(u0), s0), hmul2(e4m3x2_to_f16x2_high(u0), s0),
                                   hmul2(e4m3x2_to_f16x2(u1), s1), hmul2(e4m3x2_to_f16x2_high(u1), s1)};
#pragma unroll
            for (int j = 0; j < NT; ++j) mma_16816(o[2 * b + c][j], f, pf[mt][j][0], pf[mt][j][1]);
          }
        }
      }
      __syncwarp();   // every lane is done with the stage
      if (issued < n) {
        if (tok0 + kAtTile > end || miss != 0) fence_proxy_async_smem();
        issue(issued);
        ++issued;
      }
    }
    turn += n;
    if (!ok && n > 0) {   // given up: copies already in flight land before the CTA leaves
      for (int i = max(0, issued - kAtStages); i < issued; ++i) {
        const uint32_t bar = smem_u32(&bars[warp * kAtStages + (turn - n + i) % kAtStages]);
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(bar, ((turn - n + i) / kAtStages) & 1) && global_timer_ns() - t0 < 100000000ull) {}
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        l[j][x] += __shfl_xor_sync(0xFFFFFFFFu, l[j][x], 4);
        l[j][x] += __shfl_xor_sync(0xFFFFFFFFu, l[j][x], 8);
        l[j][x] += __shfl_xor_sync(0xFFFFFFFFu, l[j][x], 16);
      }
    // the warps' results meet in the ring: [warp][row][D], then [warp][row] of (m, l)
    __syncthreads();
    float* mo = reinterpret_cast<float*>(base);
    float2* mm = reinterpret_cast<float2*>(mo + kAtWarps * Cfg::kRows * D);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = j * 8 + 2 * t4 + x;
        if (g == 0) mm[warp * Cfg::kRows + row] = make_float2(m[j][x] == kAtNone ? -INFINITY : m[j][x], l[j][x]);
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
          *reinterpret_cast<float2*>(mo + (warp * Cfg::kRows + row) * D + c * 16 + 2 * g) = make_float2(o[c][j][x], o[c][j][x + 2]);
      }
    }
    __syncthreads();
    const bool whole_unit = tile0 == 0 && tile1 == unit_tiles;
    const int64_t part = static_cast<int64_t>(blockIdx.x) * 2 + (tile0 == 0 ? 1 : 0);
    if (tile0 == 0 && tile1 < unit_tiles) {   // goes on in the ranges up to the one with its last tile
      join.parts = (unit0 + unit_tiles - 1) / chunk - static_cast<int>(blockIdx.x) + 1;
      join.row0 = row0;
      join.n_rows = n_rows;
      join.head = head;
      join.q0 = sq.q0;
    }
    for (int i = tid; i < n_rows * (D / 2); i += kAtWarps * 32) {
      const int row = i / (D / 2), ch = (i % (D / 2)) * 2;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kAtWarps; ++w) top = fmaxf(top, mm[w * Cfg::kRows + row].x);
      float sum = 0.0f, a = 0.0f, b = 0.0f;
#pragma unroll
      for (int w = 0; w < kAtWarps; ++w) {
        const float2 ml = mm[w * Cfg::kRows + row];
        const float f = ml.x == -INFINITY ? 0.0f : ex2(ml.x - top);
        const float2 v = *reinterpret_cast<const float2*>(mo + (w * Cfg::kRows + row) * D + ch);
        sum = fmaf(ml.y, f, sum);
        a = fmaf(v.x, f, a);
        b = fmaf(v.y, f, b);
      }
      if (whole_unit) {
        const int64_t token = sq.q0 + (row0 + row) / p.group;
        const int qh = head * p.group + (row0 + row) % p.group;
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        store_attn_row(p, token, qh, D, ch, a * inv, b * inv);
        if (ch == 0 && p.lse != nullptr) p.lse[token * p.q_heads + qh] = sum > 0.0f ? (top + log2f(sum)) * 0.69314718055994531f : -INFINITY;
      } else {
        *reinterpret_cast<float2*>(p.part_o + (part * Cfg::kRows + row) * D + ch) = make_float2(a, b);
        if (ch == 0) p.part_ml[part * Cfg::kRows + row] = make_float2(top, sum);
      }
    }
    fence_proxy_async_smem();   // the ring goes back to TMA
    __syncthreads();
  }
  if (tid == 0 && p.join != nullptr) p.join[blockIdx.x] = join;
}

// Joins the parts of each unit that more than one range has, in the order of the tokens.  CTA c: the unit that starts in
// range c; its warps share the rows, and the parts of a row where there are more warps than rows.
template <int D, int NT>
__global__ void __launch_bounds__(NT * 256) attention_join_kernel(const __grid_constant__ AttnParams p) {
  constexpr int kRows = 8 * NT, V = D / 32;
  constexpr int kBatch = 8 / NT;   // parts whose loads are in flight together; by registers, as all CTAs are to run at once
  constexpr int kWarps = kRows;
  __shared__ __align__(16) float sums[kWarps][D];
  __shared__ float2 mls[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_launch_dependents();
  grid_dependency_wait();
  const AttnJoin u = p.join[blockIdx.x];
  if (u.parts <= 0) return;
  int share = 1;   // warps of a row
  while (share * 2 * u.n_rows <= kWarps) share *= 2;
  const int row = warp / share, mine = warp % share;
  if (row < u.n_rows) {
    // parts: slot 1 of this range, then slot 0 of the next ones
    float2 total = make_float2(kAtNone, 0.0f);   // reference, sum
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    for (int i0 = mine; i0 < u.parts; i0 += kBatch * share) {
      float2 ml[kBatch];
      float v[kBatch][V];
      float top = total.x;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = i0 + k * share;
        ml[k] = make_float2(-INFINITY, 0.0f);
#pragma unroll
        for (int e = 0; e < V; ++e) v[k][e] = 0.0f;
        if (i < u.parts) {
          const int64_t at = ((static_cast<int64_t>(blockIdx.x) + i) * 2 + (i == 0 ? 1 : 0)) * kRows + row;
          ml[k] = p.part_ml[at];
          const float* src = p.part_o + at * D + lane * V;
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float2 w = *reinterpret_cast<const float2*>(src + e);
            v[k][e] = w.x;
            v[k][e + 1] = w.y;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) top = fmaxf(top, ml[k].x);
      const float f0 = ex2(total.x - top);
      total = make_float2(top, total.y * f0);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] *= f0;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const float f = ex2(ml[k].x - top);   // 0 where the part saw nothing
        total.y = fmaf(ml[k].y, f, total.y);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = fmaf(v[k][e], f, acc[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < V; e += 2) *reinterpret_cast<float2*>(&sums[warp][lane * V + e]) = make_float2(acc[e], acc[e + 1]);
    if (lane == 0) mls[warp] = total;
  }
  __syncthreads();
  if (row >= u.n_rows || mine != 0) return;
  float ref = kAtNone, sum = 0.0f, acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.0f;
  for (int w = warp; w < warp + share; ++w) ref = fmaxf(ref, mls[w].x);
  for (int w = warp; w < warp + share; ++w) {
    const float f = ex2(mls[w].x - ref);
    sum = fmaf(mls[w].y, f, sum);
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = fmaf(sums[w][lane * V + e], f, acc[e]);
  }
  const int64_t token = u.q0 + (u.row0 + row) / p.group;
  const int qh = u.head * p.group + (u.row0 + row) % p.group;
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
  for (int e = 0; e < V; e += 2) store_attn_row(p, token, qh, D, lane * V + e, acc[e] * inv, acc[e + 1] * inv);
  if (lane == 0 && p.lse != nullptr) p.lse[token * p.q_heads + qh] = sum > 0.0f ? (ref + log2f(sum)) * 0.69314718055994531f : -INFINITY;
}

}  // namespace batq
