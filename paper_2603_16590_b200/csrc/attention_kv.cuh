// Attention over the paged MXFP8 key/value cache for a few query rows per key/value head (decoding, drafts).
//
//   o = sum_t softmax_t(scale * q . k_t) v_t,   k_t = 2^ek[t,b] kc[t], v_t = 2^ev[t,b] vc[t]   (b: 32-channel block)
//
// Bound by the cache's bytes: 33/32 * 2 * head_dim per token and head, read once.  Query rows of one sequence and one
// key/value head (rows = query rows x heads of the group) share every byte: a CTA takes up to 8 * NT of them and a range
// of the sequence's tokens.  Its four warps are independent of one another until the end: each has a ring of 32-token
// tiles filled by TMA, a running maximum and sum, and an accumulator; partial results of warps meet in shared memory,
// those of CTAs (a long sequence) in the workspace, in a fixed order.
//
// The products run on f16 matrix instructions (m16n8k16, fp32 sums), tokens or channels as the 16 rows and query rows as
// the 8 columns, because eight query rows would leave half of a 128-row tensor-memory tile's lanes and more unused while
// the codes would still have to be widened.  E4M3 is exact in f16; the scales are kept apart from it:
//   scores   S = sum_b 2^ek[t,b] (q_b . kc_b): one fp32 factor per token and block on the accumulators.  q is scaled by
//            a power of two per row so that its largest element is in [2^14, 2^15): exact in f16 down to 2^-31 of it.
//   values   vc 2^(ev - c) in f16 with c one integer per tile (its largest ev, less 7): exact within 2^22 of the tile's
//            largest block.  c joins the exponent of the softmax weight, w = 2^(s + c - m) with m the running maximum
//            of s + c, so that w is exact to f16 relative to the largest *contribution* to the output, not to the
//            largest probability: a token of large probability and tiny values (an attention sink) costs no precision.
//            The softmax sum takes 2^-c w in fp32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_append.cuh"
#include "ptx.cuh"

namespace batq {

constexpr int kAtWarps = 4;
constexpr int kAtTile = 32;       // tokens a warp takes at a time
constexpr int kAtStages = 3;
constexpr int kAtMinScale = -32;  // least c: an all-zero tile must not push the softmax sum's terms out of fp32

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
  int32_t row_tiles;          // of a sequence and head, at max_q
  int32_t chunk;              // tiles of 32 tokens a CTA takes
  int32_t splits;             // CTAs per row tile, at max_kv
  float* part_o;              // [unit][split][rows][head_dim]: sums relative to part_ml's reference
  float2* part_ml;            // [unit][split][rows]: reference exponent m, softmax sum
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
  static constexpr int kMult = kAtWarps * kBlocks * kAtTile * 2;
  static constexpr int kSmemBytes = kRing + kScales + kMult + 1024;
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
    s.q0 = seq;
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
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float pow2i(int e) {   // 2^e, e in [-126, 127]
  return __int_as_float((e + 127) << 23);
}
// 2^e as f16 bits; 0 below 2^-24 (e <= 7 here).
__device__ __forceinline__ uint32_t f16_pow2(int e) {
  return e >= -14 ? static_cast<uint32_t>(e + 15) << 10 : e >= -24 ? 1u << (e + 24) : 0u;
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

template <int D, int NT>
__global__ void __launch_bounds__(kAtWarps * 32) attention_kv_kernel(const __grid_constant__ CUtensorMap tmap_k,
                                                                     const __grid_constant__ CUtensorMap tmap_v,
                                                                     const __grid_constant__ AttnParams p) {
  using Cfg = AttnCfg<D, NT>;
  constexpr int BL = Cfg::kBlocks;
  extern __shared__ __align__(1024) uint8_t at_smem[];
  __shared__ __align__(8) uint64_t bars[kAtWarps * kAtStages];
  __shared__ int abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(at_smem) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = base + warp * (kAtStages * Cfg::kStageBytes);
  uint8_t* scales = base + Cfg::kRing + warp * (kAtStages * 2 * Cfg::kScaleBytes);
  uint16_t* mult = reinterpret_cast<uint16_t*>(base + Cfg::kRing + Cfg::kScales) + warp * (BL * kAtTile);

  grid_launch_dependents();
  if (lane == 0) {
    for (int i = 0; i < kAtStages; ++i) mbar_init(smem_u32(&bars[warp * kAtStages + i]), 1);
    mbar_fence_init();
  }
  if (tid == 0) abort_flag = 0;

  // this CTA's rows and tokens
  int64_t u = blockIdx.x;
  const int split = static_cast<int>(u % p.splits);
  const int64_t unit = u / p.splits;
  const int rt = static_cast<int>(unit % p.row_tiles);
  const int head = static_cast<int>(unit / p.row_tiles % p.kv_heads);
  const int seq = static_cast<int>(unit / p.row_tiles / p.kv_heads);
  grid_dependency_wait();   // q, the lengths and the cache may come from the grid in front
  const AttnSeq sq = attn_seq(p, seq);
  const int row0 = rt * Cfg::kRows, n_rows = min(Cfg::kRows, sq.nq * p.group - row0);
  if (n_rows <= 0) return;
  const int end = attn_visible(p, sq, (row0 + n_rows - 1) / p.group);   // keys the last row sees
  const int tiles = (end + kAtTile - 1) / kAtTile;
  const int tile0 = split * p.chunk, tile1 = min(tiles, tile0 + p.chunk);
  if (tile0 >= tiles && split > 0) return;
  const int used = max(1, (tiles + p.chunk - 1) / p.chunk);             // splits that have tokens

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
    m[j][0] = m[j][1] = -INFINITY;
    l[j][0] = l[j][1] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[c][j][i] = 0.0f;
  }

  // this warp's tiles: tile0 + warp + 4 i, i < n
  const int n = tile1 - tile0 > warp ? (tile1 - tile0 - warp + kAtWarps - 1) / kAtWarps : 0;
  const int32_t* pages = p.page_table + static_cast<int64_t>(seq) * p.ld_pages;
  const int page_tokens = 1 << p.page_shift;
  const int parts = page_tokens < kAtTile ? 2 : 1;   // pages of a tile
  const int part_rows = kAtTile / parts;
  // The pages of the next 32 tiles to load, one per lane (two for 16-token pages): the look-up is off the tiles' path.
  int page_a = 0, page_b = 0;
  auto look_up = [&](int i) {
    page_a = page_b = -1;
    if (i + lane < n) {
      const int tok = (tile0 + warp + kAtWarps * (i + lane)) * kAtTile;
      page_a = pages[tok >> p.page_shift];
      if (parts == 2 && tok + part_rows < end) page_b = pages[(tok + part_rows) >> p.page_shift];
    }
  };
  uint32_t bad = 0;   // bits 2 s, 2 s + 1: the first / second part of the tile in stage s is not there
  auto issue = [&](int i) {
    if ((i & 31) == 0) look_up(i);
    const int st = i % kAtStages;
    const int tok = (tile0 + warp + kAtWarps * i) * kAtTile;
    int pg[2];
    pg[0] = __shfl_sync(0xFFFFFFFFu, page_a, i & 31);
    pg[1] = __shfl_sync(0xFFFFFFFFu, page_b, i & 31);
    const uint32_t bar = smem_u32(&bars[warp * kAtStages + st]);
    uint32_t miss = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h >= parts || tok + h * part_rows >= end) continue;
      if (pg[h] < 0 || pg[h] >= p.pages) {
        miss |= 1u << h;
        if (lane == 0) atomicOr(&g_device_error, kErrorIndex);
      }
    }
    bad = (bad & ~(3u << (2 * st))) | (miss << (2 * st));
    if (lane == 0) {
      int there = 0;
      for (int h = 0; h < parts; ++h) there += tok + h * part_rows < end && !((miss >> h) & 1u);
      mbar_arrive_expect_tx(bar, there * part_rows * 2 * (D + BL));
      for (int h = 0; h < parts; ++h) {
        if (tok + h * part_rows >= end || ((miss >> h) & 1u)) continue;
        const int64_t row = ((static_cast<int64_t>(pg[h]) * p.kv_heads + head) << p.page_shift) + ((tok + h * part_rows) & (page_tokens - 1));
        const uint32_t dst = smem_u32(ring + st * Cfg::kStageBytes) + h * part_rows * D;
        tma_load_2d(dst, &tmap_k, 0, static_cast<int32_t>(row), bar);
        tma_load_2d(dst + Cfg::kCodeBytes, &tmap_v, 0, static_cast<int32_t>(row), bar);
        const uint32_t sdst = smem_u32(scales + st * 2 * Cfg::kScaleBytes) + h * part_rows * BL;
        bulk_g2s(sdst, p.k_scales + row * BL, part_rows * BL, bar);
        bulk_g2s(sdst + Cfg::kScaleBytes, p.v_scales + row * BL, part_rows * BL, bar);
      }
    }
  };
  __syncthreads();   // abort_flag
  int issued = 0;
  for (; issued < kAtStages && issued < n; ++issued) issue(issued);

  const uint32_t mult_addr = smem_u32(mult);
  bool ok = true;
  for (int i = 0; i < n; ++i) {
    const int st = i % kAtStages;
    const uint32_t bar = smem_u32(&bars[warp * kAtStages + st]);
    ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar, (i / kAtStages) & 1, &abort_flag));
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
    // the value scales of the lane's token, the tile's common exponent, and the f16 factors 2^(ev - c)
    int c_tile;
    {
      uint32_t w;
      if (BL == 4) w = *reinterpret_cast<const uint32_t*>(vs + lane * 4);
      else w = *reinterpret_cast<const uint16_t*>(vs + lane * 2);
      if (!here) w = 0;
      int top = 0;
#pragma unroll
      for (int b = 0; b < BL; ++b) top = max(top, static_cast<int>((w >> (8 * b)) & 255u));
      top = __reduce_max_sync(0xFFFFFFFFu, top);
      c_tile = max(top - 127 - 7, kAtMinScale);
      const int at = (lane & 24) | token_frag<D>(lane & 7);
#pragma unroll
      for (int b = 0; b < BL; ++b) mult[b * kAtTile + at] = static_cast<uint16_t>(f16_pow2(static_cast<int>((w >> (8 * b)) & 255u) - 127 - c_tile));
    }
    __syncwarp();

    // S^T [32 tokens x rows] in log2 units, plus c
    float s[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[mt][j][x] = 0.0f;
      const int ta = mt * 16 + frag_token<D>(g), tb = ta + 8;
      uint32_t wa, wb;
      if (BL == 4) {
        wa = *reinterpret_cast<const uint32_t*>(ks + ta * 4);
        wb = *reinterpret_cast<const uint32_t*>(ks + tb * 4);
      } else {
        wa = *reinterpret_cast<const uint16_t*>(ks + ta * 2);
        wb = *reinterpret_cast<const uint16_t*>(ks + tb * 2);
      }
#pragma unroll
      for (int b = 0; b < BL; ++b) {
        uint32_t a0, a1, b0, b1;
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(a0), "=r"(a1) : "r"(kt + tile_offset<D>(ta, 2 * b + (t4 >> 1)) + (t4 & 1) * 8) : "memory");
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(b0), "=r"(b1) : "r"(kt + tile_offset<D>(tb, 2 * b + (t4 >> 1)) + (t4 & 1) * 8) : "memory");
        const uint32_t f0[4] = {e4m3x2_to_f16x2(a0), e4m3x2_to_f16x2(b0), e4m3x2_to_f16x2_high(a0), e4m3x2_to_f16x2_high(b0)};
        const uint32_t f1[4] = {e4m3x2_to_f16x2(a1), e4m3x2_to_f16x2(b1), e4m3x2_to_f16x2_high(a1), e4m3x2_to_f16x2_high(b1)};
        const float ea = __uint_as_float(((wa >> (8 * b)) & 255u) << 23), eb = __uint_as_float(((wb >> (8 * b)) & 255u) << 23);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          mma_16816(d, f0, qf[j][b][0], qf[j][b][1]);
          mma_16816(d, f1, qf[j][b][2], qf[j][b][3]);
          s[mt][j][0] = fmaf(d[0], ea, s[mt][j][0]);
          s[mt][j][1] = fmaf(d[1], ea, s[mt][j][1]);
          s[mt][j][2] = fmaf(d[2], eb, s[mt][j][2]);
          s[mt][j][3] = fmaf(d[3], eb, s[mt][j][3]);
        }
      }
    }
    const float cf = static_cast<float>(c_tile);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          s[mt][j][x] = fmaf(s[mt][j][x], qs[j][x & 1], cf);
          if (!whole) {
            const int tt = mt * 16 + (x >> 1) * 8 + frag_token<D>(g);
            if (tok0 + tt >= lim[j][x & 1] || ((miss >> (parts == 2 ? tt >> 4 : 0)) & 1u)) s[mt][j][x] = -INFINITY;
          }
        }
    // running maximum, weights
    uint32_t pf[2][NT][2];
    const float unscale = pow2i(max(-c_tile, -126));
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float alpha[2], mr[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = fmaxf(fmaxf(s[0][j][x], s[0][j][x + 2]), fmaxf(s[1][j][x], s[1][j][x + 2]));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
        const float mn = fmaxf(m[j][x], top);
        mr[x] = mn == -INFINITY ? 0.0f : mn;
        alpha[x] = ex2(m[j][x] - mr[x]);
        m[j][x] = mn;
        float sum = 0.0f;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          s[mt][j][x] = ex2(s[mt][j][x] - mr[x]);
          s[mt][j][x + 2] = ex2(s[mt][j][x + 2] - mr[x]);
          sum += s[mt][j][x] + s[mt][j][x + 2];
        }
        l[j][x] = fmaf(l[j][x], alpha[x], sum * unscale);
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        o[c][j][0] *= alpha[0];
        o[c][j][1] *= alpha[1];
        o[c][j][2] *= alpha[0];
        o[c][j][3] *= alpha[1];
      }
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const __half2 w = __floats2half2_rn(s[mt][j][2 * h], s[mt][j][2 * h + 1]);
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
  if (!ok) {   // given up: copies already in flight land before the CTA leaves
    for (int i = max(0, issued - kAtStages); i < issued; ++i) {
      const uint32_t bar = smem_u32(&bars[warp * kAtStages + i % kAtStages]);
      const uint64_t t0 = global_timer_ns();
      while (!mbar_try_wait(bar, (i / kAtStages) & 1) && global_timer_ns() - t0 < 100000000ull) {}
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
      if (g == 0) mm[warp * Cfg::kRows + row] = make_float2(m[j][x], l[j][x]);
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
        *reinterpret_cast<float2*>(mo + (warp * Cfg::kRows + row) * D + c * 16 + 2 * g) = make_float2(o[c][j][x], o[c][j][x + 2]);
    }
  }
  __syncthreads();
  const int64_t part = unit * p.splits + split;
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
    if (used == 1) {
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
}

// Joins the splits of each row, in their order.  One warp per row of a unit.
template <int D, int NT>
__global__ void __launch_bounds__(128) attention_join_kernel(const __grid_constant__ AttnParams p, int64_t n_rows_total) {
  constexpr int kRows = 8 * NT, V = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  grid_dependency_wait();
  if (r >= n_rows_total) return;
  const int row = static_cast<int>(r % kRows);
  const int64_t unit = r / kRows;
  const int rt = static_cast<int>(unit % p.row_tiles);
  const int head = static_cast<int>(unit / p.row_tiles % p.kv_heads);
  const int seq = static_cast<int>(unit / p.row_tiles / p.kv_heads);
  const AttnSeq sq = attn_seq(p, seq);
  const int n_rows = min(kRows, sq.nq * p.group - rt * kRows);
  if (row >= n_rows) return;
  const int end = attn_visible(p, sq, (rt * kRows + n_rows - 1) / p.group);
  const int used = ((end + kAtTile - 1) / kAtTile + p.chunk - 1) / p.chunk;
  if (used <= 1) return;
  const int64_t part = unit * p.splits;
  float top = -INFINITY;
  for (int s = lane; s < used; s += 32) top = fmaxf(top, p.part_ml[(part + s) * kRows + row].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f, acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.0f;
#pragma unroll 4
  for (int s = 0; s < used; ++s) {
    const float2 ml = p.part_ml[(part + s) * kRows + row];
    const float f = ex2(ml.x - ref);   // 0 where the split saw nothing
    const float* src = p.part_o + ((part + s) * kRows + row) * D + lane * V;
    sum = fmaf(ml.y, f, sum);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 v = *reinterpret_cast<const float2*>(src + i);
      acc[i] = fmaf(v.x, f, acc[i]);
      acc[i + 1] = fmaf(v.y, f, acc[i + 1]);
    }
  }
  const int64_t token = sq.q0 + (rt * kRows + row) / p.group;
  const int qh = head * p.group + (rt * kRows + row) % p.group;
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
  for (int i = 0; i < V; i += 2) store_attn_row(p, token, qh, D, lane * V + i, acc[i] * inv, acc[i + 1] * inv);
  if (lane == 0 && p.lse != nullptr) p.lse[token * p.q_heads + qh] = sum > 0.0f ? (ref + log2f(sum)) * 0.69314718055994531f : -INFINITY;
}

}  // namespace batq
