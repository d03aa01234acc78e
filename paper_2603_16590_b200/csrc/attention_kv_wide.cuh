// Attention over the paged MXFP8 key/value cache for many query rows per key/value head (prompts and chunks of them).
//
// The same formulas as attention_kv.cuh; bound by the products, 4 * head_dim * (visible pairs) * q_heads operations, so
// they run on the 5th-generation tensor cores: tcgen05.mma kind::f16, M = 128 query rows, N = 128 tokens (scores) or
// head_dim channels (values), fp32 accumulators in tensor memory.  A unit is 256 query rows (two M tiles, rows = query
// rows x heads of the group, so that a group shares what is read and widened) of one sequence and key/value head.
//
//   tensor memory  S0 | S1 | O0 | O1, 128 columns each; the weights P (f16, two per column) overwrite their S and are the
//                  A operand of the value product from there.
//   warps 0-7      softmax: a thread owns a row.  While one M tile's warps are in their exponentials, the tensor cores can be
//                  at the other's products.  The reference follows the maximum only beyond 2^8 (as in attention_kv.cuh),
//                  so O is hardly ever read back before the end.
//   the others     one warp brings tiles, one issues the MMAs, and without READY four widen the codes: K 2^(ek - ck) and
//                  V 2^(ev - cv) in f16, ck and cv one integer per 128 tokens, into 128-byte-swizzled tiles (K: K-major B
//                  operand; V: MN-major B operand, the same bytes).  Where a token's values are more than 2^kWdEven
//                  smaller than the tile's largest, each token has its own cv, as in attention_kv.cuh: its weight
//                  would else count against the reference with the size of its neighbours' values.  Such a tile's softmax
//                  takes longer (a prompt of 8192 with nothing but such tiles 790 us instead of 500); the first one of
//                  a prompt often is one, hardly any other.  The block-scaled kinds would take the codes as they are, but want q
//                  and P in 8 bits, and V's scales along the wrong axis.
//
// What bounds it is that exponentials and products wait for one another: 256 rows x 128 tokens take 2048 cycles of the XU
// pipes (2260 as a softmax by itself) and 2048 of the tensor cores (32 MMAs of 64), and come to some 3900.  Scores ->
// weights -> P V -> the next scores is a chain within an M tile, whose S and P share a place, and P goes over only when
// all 128 columns are written.  No pipe is near its end: 1.2 instructions a cycle, XU 31 %, tensor 31 % (prompt of 2048).
// With widening warps beside it (250 instructions a tile) the softmax by itself takes 3950, so where a sequence and head
// has several units and many tiles, attention_widen_kernel writes the f16 tiles to the workspace once and this kernel copies them
// (READY): a prompt of 8192 tokens, 28 / 4 heads, takes 500 us (0.96 PFLOP/s, 0.59 of what a large bf16 product reaches)
// against 742, one of 2048, 32 / 8 heads, 71 against 82.  An item's end and the next one's start cost some 15000 cycles.
// Tried without gain: sixteen softmax warps of 64 columns (registers: the scores have to be read twice; 10000 cycles a
// tile), naps between two looks at a barrier, q of the next item brought early (1.7 % slower).
//
// Units go to the CTAs (one per SM) sequence by sequence, the longest of each first, alternately up and down.  Where there
// are few, all are divided along their tokens into as many parts as let the longest finish soonest;
// attention_wide_join_kernel adds the parts up in order.
#pragma once
#include <cstddef>
#include <type_traits>

#include "attention_kv.cuh"
#include "gemm_small_s.cuh"
#include "quantize_act_warp.cuh"

namespace batq {

constexpr int kWdRows = 256;        // of a unit
constexpr int kWdTile = 128;        // tokens
constexpr int kWdEven = 8;          // log2: weights are within 2^(kWdEven - 32) of the row's largest contribution
constexpr int kWdPartCost = 4;      // what a part of a unit costs besides its tiles, in tiles

struct AttnWidePlan { int32_t units, splits; };

// READY: the tiles come widened from the workspace (attention_widen_kernel), not from the cache.
template <int D, bool READY>
struct AttnWideShape {
  static constexpr int kThreads = READY ? 384 : 512;
  static constexpr int kStages = READY ? 4 : 3;   // f16 tiles; and of codes
  static constexpr int kIssueWarp = READY ? 8 : 12;
  // Registers of a thread of the softmax warps (which hold 128 scores), the widening ones and the others.
  static constexpr int kRegs = READY ? 168 : 128, kRegsSoftmax = READY ? 208 : 192, kRegsWiden = 80, kRegsIssue = READY ? 80 : 48;
  static_assert(256 * kRegsSoftmax + (READY ? 0 : 128 * kRegsWiden) + 128 * kRegsIssue <= kThreads * kRegs, "what the block is launched with");
};

// What the softmax has to know of a tile.
struct __align__(16) AttnTileInfo {
  int32_t ck, cv;        // the exponents that its keys and values have been divided by
  uint32_t missing;      // 16-token pieces of it whose page is not there
  int32_t uneven;        // != 0: token i's values by cv - less[i] (else less is 0)
  uint8_t less[kWdTile];
};
static_assert(sizeof(AttnTileInfo) % 16 == 0 && offsetof(AttnTileInfo, less) == 16, "copied by bulk_g2s; its head read as an int4");
// The exponent of a tile's values, or of one token's, from its largest scale byte; how much less a token's is.
__device__ __forceinline__ int attn_value_exponent(uint32_t top) { return max(static_cast<int>(top) - 127 - 7, kAtMinScale); }
__device__ __forceinline__ bool attn_uneven(uint32_t top, uint32_t low) { return attn_value_exponent(top) - attn_value_exponent(low) > kWdEven; }
__device__ __forceinline__ int attn_less(int cv, uint32_t own) { return max(cv - attn_value_exponent(own), 0); }

struct AttnWideParams {
  AttnParams a;
  uint8_t* tiles;        // READY: [sequence][head][tile][K, V], each as it stands in shared memory
  AttnTileInfo* info;    //        [sequence][head][tile]
  int32_t max_tiles;     //        of a sequence
  int32_t least_rows;   // sequences with fewer rows are attention_kv_kernel's
  int32_t max_items;    // parts of units that the workspace has room for
  AttnWidePlan* plan;   // written by the first CTA for the join; part_o, part_ml: [item][256 rows], join: [unit]
};

template <int D, bool READY>
struct AttnWideCfg {
  using Shape = AttnWideShape<D, READY>;
  static constexpr int kBlocks = D / 32;
  static constexpr int kPanels = D / 64;                         // 64-channel halves of a row: 128 bytes of f16
  static constexpr int kHalfTile = 128 * 128;                    // 128 rows of one panel
  static constexpr int kQBytes = 2 * kPanels * kHalfTile;        // two M tiles
  static constexpr int kF16Bytes = kPanels * kHalfTile;          // one widened tile
  static constexpr int kCodeBytes = kWdTile * D;
  static constexpr int kScaleBytes = kWdTile * kBlocks;          // of K or V
  static constexpr int kScaleSlots = 4;
  static constexpr int kF16At = kQBytes, kCodeAt = kF16At + Shape::kStages * kF16Bytes, kScaleAt = kCodeAt + Shape::kStages * kCodeBytes;
  static constexpr int kSmemBytes = (READY ? kCodeAt : kScaleAt + kScaleSlots * 2 * kScaleBytes) + 1024;
};

// As f16_idesc_bf16 with f16 operands; b_mn: B is MN-major.
__host__ __device__ constexpr uint32_t f16_idesc_f16(int M, int N, bool b_mn) {
  return (1u << 4) | (b_mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ void tc_mma_f16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
// Waits for the loads in front; the registers that one of them fills are named so that nothing that uses them can be
// moved ahead of the wait.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint32_t f16x2_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// One part of a unit.
struct AttnWideItem {
  AttnSeq sq;
  int seq, head, row0, n_rows, unit, split;
  int end;             // keys that the unit's last row sees
  int tile0, tile1;
};

template <int D, bool READY>
__global__ void __launch_bounds__(AttnWideShape<D, READY>::kThreads, 1)
attention_kv_wide_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                         const __grid_constant__ AttnWideParams wp) {
  using Cfg = AttnWideCfg<D, READY>;
  using Shape = AttnWideShape<D, READY>;
  constexpr int BL = Cfg::kBlocks, kStages = Shape::kStages;
  const AttnParams& p = wp.a;
  extern __shared__ __align__(1024) uint8_t wd_smem[];
  __shared__ __align__(8) uint64_t code_full[kStages], code_empty[kStages], f16_full[kStages], f16_empty[kStages];
  __shared__ __align__(8) uint64_t s_full[2], p_ready[2], o_done[2], q_ready[2], drain;
  __shared__ int first[kAtMaxSeqs];   // units in front of each sequence's
  __shared__ int scan_sum[Shape::kThreads / 32], scan_max[Shape::kThreads / 32];
  __shared__ __align__(16) AttnTileInfo info[Cfg::kScaleSlots];
  // 2^(e - c) of a tile's keys, values: f16, [block][token % 8][token / 8], so that a widening thread's are one run
  __shared__ __align__(16) uint16_t factors[READY ? 1 : 2][READY ? 1 : kWdTile * BL];
  __shared__ uint32_t tmem_base_smem;
  __shared__ int abort_flag;
  __shared__ volatile int widen_stop;   // a widening warp's wait has run out
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(wd_smem) + 1023) & ~uintptr_t(1023));

  grid_launch_dependents();
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&code_full[i]), 1);
      mbar_init(smem_u32(&code_empty[i]), 4);
      mbar_init(smem_u32(&f16_full[i]), READY ? 1 : 4);
      mbar_init(smem_u32(&f16_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s_full[i]), 1);
      mbar_init(smem_u32(&p_ready[i]), 4);
      mbar_init(smem_u32(&o_done[i]), 1);
      mbar_init(smem_u32(&q_ready[i]), 4);
    }
    mbar_init(smem_u32(&drain), 1);
    mbar_fence_init();
    abort_flag = 0;
    widen_stop = 0;
    if (!READY) {
      tma_prefetch_desc(&tmap_k);
      tma_prefetch_desc(&tmap_v);
    }
  }
  grid_dependency_wait();   // q, the lengths and the cache may come from the grid in front
  if (warp == Shape::kIssueWarp + 1) {   // not before: the grid in front may still want tensor memory of this SM
    tmem_alloc(smem_u32(&tmem_base_smem), 512);
    tmem_relinquish();
  }

  // units of each sequence, of all, and the most tiles of one
  int units, splits;
  {
    int mine[2] = {0, 0}, tiles = 0;   // two sequences a thread
    static_assert(kAtMaxSeqs <= 2 * 256, "");
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int s = 2 * tid + i;
      if (s < p.seqs) {
        const AttnSeq q = attn_seq(p, s);
        const int rows = q.nq * p.group;
        mine[i] = rows >= wp.least_rows ? p.kv_heads * ((rows + kWdRows - 1) / kWdRows) : 0;
        if (mine[i] > 0) tiles = max(tiles, (q.len + kWdTile - 1) / kWdTile);
      }
    }
    int scan = mine[0] + mine[1];
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, scan, x);
      if (lane >= x) scan += v;
    }
    tiles = __reduce_max_sync(0xFFFFFFFFu, tiles);
    if (lane == 31) scan_sum[warp] = scan;
    if (lane == 0) scan_max[warp] = tiles;
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    int before = scan - mine[0] - mine[1];
    units = tiles = 0;
    for (int w = 0; w < Shape::kThreads / 32; ++w) {
      if (w < warp) before += scan_sum[w];
      units += scan_sum[w];
      tiles = max(tiles, scan_max[w]);
    }
    if (2 * tid < kAtMaxSeqs) {
      first[2 * tid] = before;
      first[2 * tid + 1] = before + mine[0];
    }
    __syncthreads();
    splits = 1;
    int best = INT_MAX;
    const int grid = static_cast<int>(gridDim.x);
    for (int c = 1; units > 0 && c <= tiles && static_cast<int64_t>(units) * c <= wp.max_items; ++c) {
      const int cost = (units * c + grid - 1) / grid * ((tiles + c - 1) / c + kWdPartCost);
      if (cost < best) { best = cost; splits = c; }
    }
  }
  const int items = units * splits;
  if (tid == 0 && blockIdx.x == 0 && wp.plan != nullptr) *wp.plan = AttnWidePlan{units, splits};
  const uint32_t tmem = 0;   // all 512 columns are this CTA's

  // the k-th item of this CTA; false: there is none
  auto item_at = [&](int k, AttnWideItem* it) {
    const int grid = static_cast<int>(gridDim.x), b = static_cast<int>(blockIdx.x);
    const int64_t at = static_cast<int64_t>(k) * grid + ((k & 1) ? grid - 1 - b : b);
    if (at >= items) return false;
    const int i = static_cast<int>(at);
    it->unit = splits == 1 ? i : i / splits;
    it->split = i - it->unit * splits;
    int lo = 0, hi = p.seqs - 1;   // the last sequence that starts at or before the unit
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= it->unit) lo = mid;
      else hi = mid - 1;
    }
    it->seq = lo;
    it->sq = attn_seq(p, lo);
    const int rows = it->sq.nq * p.group, row_tiles = (rows + kWdRows - 1) / kWdRows, local = it->unit - first[lo];
    const int up = local / p.kv_heads;
    it->head = local - up * p.kv_heads;
    it->row0 = (row_tiles - 1 - up) * kWdRows;
    it->n_rows = min(kWdRows, rows - it->row0);
    it->end = attn_visible(p, it->sq, (it->row0 + it->n_rows - 1) / p.group);
    const int tiles = (it->end + kWdTile - 1) / kWdTile;   // times the parts of a unit: below 2^31
    it->tile0 = splits == 1 ? 0 : tiles * it->split / splits;
    it->tile1 = splits == 1 ? tiles : tiles * (it->split + 1) / splits;
    return true;
  };

  AttnWideItem it;
  if (warp < 8) {
    // ------------------------------------------------------------------ softmax: thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Shape::kRegsSoftmax));
    const int g = warp >> 2, r = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;   // tensor memory lanes of this warp
    const uint32_t s_at = tmem + lanes + g * 128, o_at = tmem + lanes + 256 + g * 128;
    uint8_t* qt = base + g * (Cfg::kQBytes / 2) + r * 128;
    uint32_t s_phase = 0, o_phase = 0;
    int turn = 0;   // tiles of the CTA in front of this item's: index of exponents, missing
    bool ok = true;
    for (int k = 0; ok && item_at(k, &it); ++k) {
      const int row = it.row0 + g * 128 + r;
      const bool real = g * 128 + r < it.n_rows, active = g * 128 < it.n_rows;
      const int qi = row / p.group, qh = it.head * p.group + row % p.group;
      const int64_t token = it.sq.q0 + qi;
      const int n = it.tile1 - it.tile0;
      // q in f16, scaled so that the row's largest element is in [2^14, 2^15); the sign of the scale goes with it
      float qs = 0.0f;
      if (active && n > 0) {
        // The warp brings its 32 rows as they are, whole rows at a time, to where they will stand in f16; then each
        // thread turns its own.
        const int64_t q_off = token * p.ldq + static_cast<int64_t>(qh) * D;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const int at = i * (256 / D) + lane / (D / 8), ch = lane % (D / 8), rr = (warp & 3) * 32 + at;
          const int64_t off = __shfl_sync(0xFFFFFFFFu, q_off, at);
          const bool there = __shfl_sync(0xFFFFFFFFu, real, at);
          cp_async_16(smem_u32(base + g * (Cfg::kQBytes / 2) + rr * 128 + (ch >> 3) * Cfg::kHalfTile + (((ch & 7) ^ (rr & 7)) << 4)),
                      p.q + (there ? off : 0) + ch * 8, there ? 16 : 0);
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncwarp();
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          float v[8];
          unpack_bf16x8(*reinterpret_cast<const uint4*>(qt + (i >> 3) * Cfg::kHalfTile + (((i & 7) ^ (r & 7)) << 4)), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
        }
        const int e = max(static_cast<int>(__float_as_uint(amax) >> 23) - 127, -100);
        const float up = p.scale_log2 < 0.0f ? -pow2i(14 - e) : pow2i(14 - e);
        qs = fmaxf(fabsf(p.scale_log2) * pow2i(e - 14), 1e-37f);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          uint4* at = reinterpret_cast<uint4*>(qt + (i >> 3) * Cfg::kHalfTile + (((i & 7) ^ (r & 7)) << 4));
          float v[8];
          unpack_bf16x8(*at, v);
          *at = make_uint4(f16x2_pack(v[0] * up, v[1] * up), f16x2_pack(v[2] * up, v[3] * up), f16x2_pack(v[4] * up, v[5] * up),
                           f16x2_pack(v[6] * up, v[7] * up));
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();   // what was read of tensor memory for the item before
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&q_ready[g]));
      }

      const int lim = real ? attn_visible(p, it.sq, qi) : 0;            // keys this row sees
      const int full = attn_visible(p, it.sq, it.row0 / p.group);       // keys that every row sees
      float m = kAtNone, l = 0.0f;
      for (int j = 0; active && j < n; ++j) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(smem_u32(&s_full[g]), s_phase, &abort_flag));
        if (!ok) break;
        s_phase ^= 1u;
        tc_fence_after_sync();
        const AttnTileInfo& tile = info[(turn + j) % Cfg::kScaleSlots];
        const int4 ex = *reinterpret_cast<const int4*>(&tile);   // ck, cv, missing, uneven
        const uint32_t miss = static_cast<uint32_t>(ex.z);
        const bool uneven = ex.w != 0;
        const int tok0 = (it.tile0 + j) * kWdTile, see = lim - tok0;
        const bool part = tok0 + kWdTile > full || miss != 0;
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(s_at + c * 32, s[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_wait_for(s[c]);
        if (part) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c * 32 + i >= see) s[c][i] = 0xFF800000u;
          if (miss != 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if ((miss >> (c * 2 + (i >> 4))) & 1u) s[c][i] = 0xFF800000u;
          }
        }
        float qk = fmaxf(qs * pow2i(max(ex.x, -126)), 1e-37f);
        const float cv = static_cast<float>(ex.y);
        if (uneven) {   // each token's score with its own exponent, relative to the tile's
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const uchar4 d = *reinterpret_cast<const uchar4*>(&tile.less[c * 32 + i]);
              s[c][i] = __float_as_uint(fmaf(__uint_as_float(s[c][i]), qk, -static_cast<float>(d.x)));
              s[c][i + 1] = __float_as_uint(fmaf(__uint_as_float(s[c][i + 1]), qk, -static_cast<float>(d.y)));
              s[c][i + 2] = __float_as_uint(fmaf(__uint_as_float(s[c][i + 2]), qk, -static_cast<float>(d.z)));
              s[c][i + 3] = __float_as_uint(fmaf(__uint_as_float(s[c][i + 3]), qk, -static_cast<float>(d.w)));
            }
          qk = 1.0f;
        }
        float tops[4];   // four chains: one takes 10 cycles a step
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tops[c] = __uint_as_float(s[c][0]);
#pragma unroll
          for (int i = 1; i < 32; ++i) tops[c] = fmaxf(tops[c], __uint_as_float(s[c][i]));
        }
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        if (__any_sync(0xFFFFFFFFu, fmaf(top, qk, cv - m) > kAtMost)) {
          const float mn = fmaxf(m, fmaf(top, qk, cv) - kAtHead), alpha = ex2(m - mn);
          m = mn;
          l *= alpha;
          if (j > 0) {   // the value product of the tile before is done: its S was waited for
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
              uint32_t o[16];
              tmem_ld_32x32b_x16(o_at + c * 16, o);
              tmem_ld_wait_for(o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              tmem_st_32x32b_x16(o_at + c * 16, o);
            }
          }
        }
        const uint64_t qk2 = f32x2_pack(qk, qk), t2 = f32x2_pack(cv - m, cv - m);
        uint64_t sum0 = 0, sum1 = 0;
        auto weigh = [&](auto per_token) {   // the weights, to where the scores were, and their sum
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t (&x)[32] = s[c];
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float a, b;
              f32x2_unpack(f32x2_fma(f32x2_pack(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), qk2, t2), a, b);
              a = ex2(a);
              b = ex2(b);
              uint64_t& sum = i & 1 ? sum1 : sum0;
              if (per_token.value) {
                const uchar2 d = *reinterpret_cast<const uchar2*>(&tile.less[c * 32 + 2 * i]);
                sum = f32x2_fma(f32x2_pack(a, b), f32x2_pack(pow2i(d.x - ex.y), pow2i(d.y - ex.y)), sum);
              } else {
                sum = f32x2_add(sum, f32x2_pack(a, b));
              }
              w[i] = f16x2_pack(a, b);
            }
            tmem_st_32x32b_x16(s_at + c * 16, w);
          }
        };
        if (uneven) weigh(std::true_type{});
        else weigh(std::false_type{});
        float a, b;
        f32x2_unpack(f32x2_add(sum0, sum1), a, b);
        l = fmaf(a + b, uneven ? 1.0f : pow2i(-ex.y), l);
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&p_ready[g]));
      }
      if (!ok) break;
      turn += n;
      if (!active) continue;
      if (n > 0) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(smem_u32(&o_done[g]), o_phase, &abort_flag));
        if (!ok) break;
        o_phase ^= 1u;
        tc_fence_after_sync();
      }
      const bool seen = m != kAtNone;
      const float inv = seen && l > 0.0f ? 1.0f / l : 0.0f;
      const int64_t part = (static_cast<int64_t>(it.unit) * splits + it.split) * kWdRows + g * 128 + r;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        __syncwarp();
        if (n > 0) {
          tmem_ld_32x32b_x32(o_at + c * 32, o);
          tmem_ld_wait_for(o);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (n == 0 || !seen) o[i] = 0u;
        if (splits == 1) {   // to the row's place in the M tile of q, which no MMA reads any more
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(o[8 * i + 2 * h]) * inv, __uint_as_float(o[8 * i + 2 * h + 1]) * inv);
              w[h] = *reinterpret_cast<const uint32_t*>(&v);
            }
            const int ch = c * 4 + i;
            *reinterpret_cast<uint4*>(qt + (ch >> 3) * Cfg::kHalfTile + (((ch & 7) ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else if (real) {
          uint4* dst = reinterpret_cast<uint4*>(p.part_o + part * D + c * 32);
#pragma unroll
          for (int i = 0; i < 8; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
      }
      if (splits == 1) {   // whole rows at a time
        __syncwarp();
        const int64_t o_off = token * p.ldo + static_cast<int64_t>(qh) * D;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const int at = i * (256 / D) + lane / (D / 8), ch = lane % (D / 8), rr = (warp & 3) * 32 + at;
          const int64_t off = __shfl_sync(0xFFFFFFFFu, o_off, at);
          const uint4 v = *reinterpret_cast<const uint4*>(base + g * (Cfg::kQBytes / 2) + rr * 128 + (ch >> 3) * Cfg::kHalfTile + (((ch & 7) ^ (rr & 7)) << 4));
          if (__shfl_sync(0xFFFFFFFFu, real, at)) *reinterpret_cast<uint4*>(p.out + off + ch * 8) = v;
        }
        __syncwarp();
      }
      if (real && splits == 1 && p.lse != nullptr) p.lse[token * p.q_heads + qh] = inv > 0.0f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
      if (real && splits > 1) p.part_ml[part] = make_float2(seen ? m : -INFINITY, l);
      if (splits > 1 && it.split == 0 && tid == 0) p.join[it.unit] = AttnJoin{splits, it.row0, it.n_rows, it.head, it.sq.q0};
    }
  } else if (!READY && warp < 12) {
    // ------------------------------------------------------------------ codes -> f16
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegsWiden));
    // A thread widens sixteen codes (eight with D = 64) of every eighth token, always the same channels: its rows stand
    // alike in the swizzle, so that addresses only advance, and neither the reads nor the writes of a warp meet in a
    // bank.  Shared-memory instructions queue behind the exponentials of the softmax warps: there are as few as can be.
    constexpr int kCodes = D / 8, kRowsStep = 8;
    const int ct = tid - 256, c = ct & 7, r0 = ct >> 3, b = c * kCodes / 32, half = r0 >> 3;   // rows r0 % 8 + 8 i, i of the thread's half
    const int row_first = (r0 & 7) + half * 64;
    const int code_at = D == 128 ? tile_offset<128>(row_first, c) : tile_offset<64>(row_first, c >> 1) + (c & 1) * 8;
    const int ch0 = c * kCodes;   // first channel
    const int f16_at = (ch0 >> 6) * Cfg::kHalfTile + row_first * 128;
    const int x0 = (((ch0 >> 3) & 7) ^ (r0 & 7)) << 4, x1 = ((((ch0 >> 3) + 1) & 7) ^ (r0 & 7)) << 4;   // its 16-byte pieces
    const bool swap = D == 128 && (c & 4) != 0;   // lanes of the second panel write theirs in the other order
    uint32_t n_step = 0;   // K and V tiles of the CTA so far: stage n_step % kStages
    int turn = 0;
    bool ok = true;
    for (int k = 0; ok && item_at(k, &it); ++k) {
      for (int t = it.tile0; ok && t < it.tile1; ++t, ++turn) {
        const int slot = turn % Cfg::kScaleSlots, there = it.end - t * kWdTile;   // tokens of the tile that count
        const uint8_t* ks = base + Cfg::kScaleAt + slot * 2 * Cfg::kScaleBytes;
        const uint8_t* vs = ks + Cfg::kScaleBytes;
        int cs[2];
        uint32_t miss = 0;
        bool cut = false, uneven = false;
#pragma unroll
        for (int v = 0; v < 2; ++v, ++n_step) {   // K, then V
          const uint32_t st = n_step % kStages, phase = (n_step / kStages) & 1u;
          const bool got = __all_sync(0xFFFFFFFFu, mbar_wait_short(smem_u32(&code_full[st]), phase, &abort_flag) &&
                                                       mbar_wait_short(smem_u32(&f16_empty[st]), phase ^ 1u, &abort_flag));
          // The four warps leave together: one that went by its own wait would be missed at the barriers below, whose
          // waits have no limit.  The flag is written in front of the first or behind the second, and read in between.
          if (!got && lane == 0) widen_stop = 1;
          if (v == 0) {
            // (the tile before is widened everywhere: its factors go)
            named_barrier_sync(1, 128);
            ok = widen_stop == 0;
            if (!ok) break;
            // the tile's exponents, in every warp (a lane has four tokens), then the factors of the thread's own token
            miss = info[slot].missing;
            cut = there < kWdTile || miss != 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint8_t* src = x == 0 ? ks : vs;
              uint32_t top = 0, low = 255;   // the largest byte of the tile; the least of the tokens' largest (of the values)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t w = largest_byte(BL == 4 ? *reinterpret_cast<const uint32_t*>(src + (4 * lane + i) * 4)
                                                        : *reinterpret_cast<const uint16_t*>(src + (4 * lane + i) * 2));
                if (!cut || (4 * lane + i < there && !((miss >> (lane >> 2)) & 1u))) {
                  top = max(top, w);
                  low = min(low, w);
                }
              }
              top = __reduce_max_sync(0xFFFFFFFFu, top);
              int c_own = x == 0 ? max(static_cast<int>(top) - 127 - 7, -100) : attn_value_exponent(top);
              cs[x] = c_own;
              const uint32_t w = BL == 4 ? *reinterpret_cast<const uint32_t*>(src + ct * 4) : *reinterpret_cast<const uint16_t*>(src + ct * 2);
              if (x == 1) {
                uneven = attn_uneven(top, __reduce_min_sync(0xFFFFFFFFu, low));
                const int less = uneven ? attn_less(c_own, largest_byte(w)) : 0;
                c_own -= less;
                info[slot].less[ct] = static_cast<uint8_t>(less);
              }
#pragma unroll
              for (int h = 0; h < BL / 2; ++h) {
                uint32_t f = f16_pow2x2(__byte_perm(w, 0u, h == 0 ? 0x4140 : 0x4342), c_own + 127);
                // behind the last key (or on a page that is not there) anything may stand: values count as zero
                if (x == 1 && cut && (ct >= there || ((miss >> (ct >> 4)) & 1u))) f = 0u;
                uint16_t* at = &factors[READY ? 0 : x][2 * h * kWdTile + (ct & 7) * 16 + (ct >> 3)];
                at[0] = static_cast<uint16_t>(f);
                at[kWdTile] = static_cast<uint16_t>(f >> 16);
              }
            }
            if (ct == 0) { info[slot].ck = cs[0]; info[slot].cv = cs[1]; info[slot].uneven = uneven; }
            named_barrier_sync(1, 128);
          }
          if (!got) continue;   // (the values': on to the next tile's first barrier, if there is one)
          const uint8_t* codes = base + Cfg::kCodeAt + st * Cfg::kCodeBytes + code_at;
          uint8_t* dst = base + Cfg::kF16At + st * Cfg::kF16Bytes + f16_at;
          const uint4 fs = *reinterpret_cast<const uint4*>(&factors[READY ? 0 : v][b * kWdTile + (r0 & 7) * 16 + half * 8]);
          const uint32_t fw[4] = {fs.x, fs.y, fs.z, fs.w};
          auto widen = [&](auto check) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t f = __byte_perm(fw[i >> 1], 0u, (i & 1) ? 0x3232 : 0x1010);
              uint8_t* line = dst + i * kRowsStep * 128;
              if (D == 128) {
                uint4 w = *reinterpret_cast<const uint4*>(codes + i * kRowsStep * D);
                if (check.value && f == 0u) w = make_uint4(0u, 0u, 0u, 0u);   // not NaN times zero
                if (swap) { uint32_t t = w.x; w.x = w.z; w.z = t; t = w.y; w.y = w.w; w.w = t; }
                *reinterpret_cast<uint4*>(line + (swap ? x1 : x0)) = make_uint4(hmul2(e4m3x2_to_f16x2(w.x), f), hmul2(e4m3x2_to_f16x2_high(w.x), f),
                                                                              hmul2(e4m3x2_to_f16x2(w.y), f), hmul2(e4m3x2_to_f16x2_high(w.y), f));
                *reinterpret_cast<uint4*>(line + (swap ? x0 : x1)) = make_uint4(hmul2(e4m3x2_to_f16x2(w.z), f), hmul2(e4m3x2_to_f16x2_high(w.z), f),
                                                                              hmul2(e4m3x2_to_f16x2(w.w), f), hmul2(e4m3x2_to_f16x2_high(w.w), f));
              } else {
                uint2 w = *reinterpret_cast<const uint2*>(codes + i * kRowsStep * D);
                if (check.value && f == 0u) w = make_uint2(0u, 0u);
                *reinterpret_cast<uint4*>(line + x0) = make_uint4(hmul2(e4m3x2_to_f16x2(w.x), f), hmul2(e4m3x2_to_f16x2_high(w.x), f),
                                                                 hmul2(e4m3x2_to_f16x2(w.y), f), hmul2(e4m3x2_to_f16x2_high(w.y), f));
              }
            }
          };
          if (v == 1 && cut) widen(std::true_type{});
          else widen(std::false_type{});
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(smem_u32(&code_empty[st]));
            mbar_arrive(smem_u32(&f16_full[st]));
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegsIssue));
    if (READY && warp == Shape::kIssueWarp) {
      // ---------------------------------------------------------------- widened tiles, 32 KB (16 KB) a copy
      uint32_t n_step = 0;
      int turn = 0;
      bool ok = true;
      for (int k = 0; ok && item_at(k, &it); ++k) {
        const int64_t line = (static_cast<int64_t>(it.seq) * p.kv_heads + it.head) * wp.max_tiles;
        for (int t = it.tile0; ok && t < it.tile1; ++t, ++turn) {
#pragma unroll
          for (int v = 0; v < 2; ++v, ++n_step) {
            const uint32_t st = n_step % kStages, phase = (n_step / kStages) & 1u;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(smem_u32(&f16_empty[st]), phase ^ 1u, &abort_flag));
            if (!ok) break;
            if (lane == 0) {
              const uint32_t bar = smem_u32(&f16_full[st]);
              mbar_arrive_expect_tx(bar, Cfg::kF16Bytes + (v == 0 ? static_cast<int>(sizeof(AttnTileInfo)) : 0));
              if (v == 0) bulk_g2s(smem_u32(&info[turn % Cfg::kScaleSlots]), wp.info + line + t, sizeof(AttnTileInfo), bar);
              bulk_g2s(smem_u32(base + Cfg::kF16At + st * Cfg::kF16Bytes), wp.tiles + ((line + t) * 2 + v) * Cfg::kF16Bytes, Cfg::kF16Bytes, bar);
            }
            __syncwarp();
          }
        }
      }
      // copies in flight land before the CTA leaves: whoever waits for the last ones may have given up
      for (uint32_t i = n_step > kStages ? n_step - kStages : 0; i < n_step; ++i) {
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(smem_u32(&f16_full[i % kStages]), (i / kStages) & 1u) && global_timer_ns() - t0 < 100000000ull) {}
      }
    } else if (!READY && warp == Shape::kIssueWarp) {
      // ---------------------------------------------------------------- codes and scales by TMA
      const int box = min(1 << p.page_shift, 32), boxes = kWdTile / box;   // rows of a copy; copies of a tile
      uint32_t n_step = 0;
      int turn = 0;
      bool ok = true;
      for (int k = 0; ok && item_at(k, &it); ++k) {
        const int32_t* pages = p.page_table + static_cast<int64_t>(it.seq) * p.ld_pages;
        auto look_up = [&](int t) {   // lane = copy
          const int tok = t * kWdTile + lane * box;
          return lane < boxes && t < it.tile1 && tok < it.end ? pages[tok >> p.page_shift] : -1;
        };
        int next = look_up(it.tile0);
        for (int t = it.tile0; ok && t < it.tile1; ++t, ++turn) {
          const int page = next, slot = turn % Cfg::kScaleSlots;
          next = look_up(t + 1);
          const int tok = t * kWdTile + lane * box;
          const bool wanted = lane < boxes && tok < it.end;
          const bool have = wanted && static_cast<uint32_t>(page) < static_cast<uint32_t>(p.pages);
          const uint32_t lost = __ballot_sync(0xFFFFFFFFu, wanted && !have);
          const int n_have = __popc(__ballot_sync(0xFFFFFFFFu, have));
          const int row = ((page * p.kv_heads + it.head) << p.page_shift) + (tok & ((1 << p.page_shift) - 1));   // below 2^31
#pragma unroll
          for (int v = 0; v < 2; ++v, ++n_step) {
            const uint32_t st = n_step % kStages, phase = (n_step / kStages) & 1u;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(smem_u32(&code_empty[st]), phase ^ 1u, &abort_flag));
            if (!ok) break;
            const uint32_t bar = smem_u32(&code_full[st]);
            if (lane == 0) {
              if (v == 0) {
                uint32_t miss = 0;
                for (int i = 0; i < boxes; ++i)
                  if ((lost >> i) & 1u) miss |= (box == 32 ? 3u : 1u) << (i * (box / 16));
                info[slot].missing = miss;
                if (miss != 0) atomicOr(&g_device_error, kErrorIndex);
              }
              mbar_arrive_expect_tx(bar, n_have * box * (D + (v == 0 ? 2 * BL : 0)));
            }
            __syncwarp();
            if (have) {
              const uint32_t dst = smem_u32(base + Cfg::kCodeAt + st * Cfg::kCodeBytes) + lane * box * D;
              if (v == 0) {
                const uint32_t sdst = smem_u32(base + Cfg::kScaleAt + slot * 2 * Cfg::kScaleBytes) + lane * box * BL;
                tma_load_2d(dst, &tmap_k, 0, row, bar);
                bulk_g2s(sdst, p.k_scales + static_cast<int64_t>(row) * BL, box * BL, bar);
                bulk_g2s(sdst + Cfg::kScaleBytes, p.v_scales + static_cast<int64_t>(row) * BL, box * BL, bar);
              } else {
                tma_load_2d(dst, &tmap_v, 0, row, bar);
              }
            }
            __syncwarp();
          }
        }
      }
      // copies in flight land before the CTA leaves: whoever waits for the last ones may have given up
      for (uint32_t i = n_step > kStages ? n_step - kStages : 0; i < n_step; ++i) {
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(smem_u32(&code_full[i % kStages]), (i / kStages) & 1u) && global_timer_ns() - t0 < 100000000ull) {}
      }
    } else if (warp == Shape::kIssueWarp + 1) {
      // ---------------------------------------------------------------- MMAs
      constexpr uint32_t idesc_s = f16_idesc_f16(128, kWdTile, false), idesc_o = f16_idesc_f16(128, D, true);
      const uint64_t q_desc = make_smem_desc(smem_u32(base), 16, 1024, 2);                              // K-major, 128-byte swizzle
      const uint64_t k_desc = make_smem_desc(smem_u32(base + Cfg::kF16At), 16, 1024, 2);
      const uint64_t v_desc = make_smem_desc(smem_u32(base + Cfg::kF16At), Cfg::kHalfTile, 1024, 2);    // MN-major: panels, 8 tokens
      uint32_t n_step = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t phase) {
        ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait_short(smem_u32(bar), phase, &abort_flag));
        return ok;
      };
      auto scores = [&](int g, uint32_t st) {
        const uint64_t a = q_desc + static_cast<uint32_t>((g * (Cfg::kQBytes / 2)) >> 4);
        const uint64_t b = k_desc + static_cast<uint32_t>((st * Cfg::kF16Bytes) >> 4);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = static_cast<uint32_t>(((kk >> 2) * Cfg::kHalfTile + (kk & 3) * 32) >> 4);
            tc_mma_f16(tmem + g * 128, a + off, b + off, idesc_s, kk > 0);
          }
          tc_commit(smem_u32(&s_full[g]));
        }
        __syncwarp();
      };
      for (int k = 0; ok && item_at(k, &it); ++k) {
        const int n = it.tile1 - it.tile0, groups = it.n_rows > 128 ? 2 : 1;
        if (n <= 0) continue;
        for (int g = 0; g < groups && wait(&q_ready[g], q_phase[g]); ++g) q_phase[g] ^= 1u;
        if (!ok) break;
        // step of tile j: K n_step + 2 j, V n_step + 2 j + 1
        if (!wait(&f16_full[n_step % kStages], (n_step / kStages) & 1u)) break;
        tc_fence_after_sync();
        for (int g = 0; g < groups; ++g) scores(g, n_step % kStages);
        if (elect_one()) tc_commit(smem_u32(&f16_empty[n_step % kStages]));
        __syncwarp();
        for (int j = 0; ok && j < n; ++j) {
          const uint32_t vn = n_step + 2 * j + 1, kn = vn + 1, vst = vn % kStages, kst = kn % kStages;
          // These are here long before the weights are, and asking for them takes some 400 cycles: not between products.
          if (!wait(&f16_full[vst], (vn / kStages) & 1u)) break;
          if (j + 1 < n && !wait(&f16_full[kst], (kn / kStages) & 1u)) break;
          for (int g = 0; g < groups; ++g) {
            if (!wait(&p_ready[g], p_phase[g])) break;
            p_phase[g] ^= 1u;
            tc_fence_after_sync();
            if (elect_one()) {
              const uint64_t v = v_desc + static_cast<uint32_t>((vst * Cfg::kF16Bytes) >> 4);
#pragma unroll
              for (int kk = 0; kk < kWdTile / 16; ++kk)
                tc_mma_f16_ta(tmem + 256 + g * 128, tmem + g * 128 + kk * 8, v + static_cast<uint32_t>((kk * 2048) >> 4), idesc_o, j > 0 || kk > 0);
              if (g == groups - 1) tc_commit(smem_u32(&f16_empty[vst]));
              if (j == n - 1) tc_commit(smem_u32(&o_done[g]));
            }
            __syncwarp();
            if (j + 1 < n) {
              scores(g, kst);
              if (g == groups - 1) {
                if (elect_one()) tc_commit(smem_u32(&f16_empty[kst]));
                __syncwarp();
              }
            }
          }
        }
        n_step += 2 * n;
      }
      // whatever was issued is over before tensor memory goes back
      if (elect_one()) tc_commit(smem_u32(&drain));
      __syncwarp();
      const uint64_t t0 = global_timer_ns();
      while (!mbar_try_wait(smem_u32(&drain), 0) && global_timer_ns() - t0 < kWaitLimitNs) {}
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == Shape::kIssueWarp + 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base_smem, 512);
  }
}

// K and V of the sequences that attention_kv_wide_kernel takes, widened once for all its units: CTA (tile, head, sequence)
// writes the two f16 tiles as they will stand in shared memory, and their AttnTileInfo.
template <int D>
__global__ void __launch_bounds__(128) attention_widen_kernel(const __grid_constant__ AttnWideParams wp, const uint8_t* __restrict__ k_codes,
                                                              const uint8_t* __restrict__ v_codes) {
  using Cfg = AttnWideCfg<D, true>;
  constexpr int BL = Cfg::kBlocks, kChunks = D / 16;   // 16-code chunks of a row
  const AttnParams& p = wp.a;
  __shared__ int rows[kWdTile];                    // a token's row of the pool, -1: none
  __shared__ uint16_t factors[2][kWdTile * BL];
  __shared__ uint32_t tops[2][4], lows[4], lost[4];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t = blockIdx.x, head = blockIdx.y, seq = blockIdx.z;
  grid_launch_dependents();
  grid_dependency_wait();
  const AttnSeq sq = attn_seq(p, seq);
  if (sq.nq * p.group < wp.least_rows || t * kWdTile >= sq.len) return;
  const int tok = t * kWdTile + tid;
  int row = -1;
  bool miss = false;
  if (tok < sq.len) {
    const int page = p.page_table[static_cast<int64_t>(seq) * p.ld_pages + (tok >> p.page_shift)];
    miss = static_cast<uint32_t>(page) >= static_cast<uint32_t>(p.pages);
    if (!miss) row = ((page * p.kv_heads + head) << p.page_shift) + (tok & ((1 << p.page_shift) - 1));   // below 2^31
  }
  rows[tid] = row;
  uint32_t w[2] = {0u, 0u};   // the token's scale bytes
  if (row >= 0) {
    if (BL == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p.k_scales + static_cast<int64_t>(row) * 4);
      w[1] = *reinterpret_cast<const uint32_t*>(p.v_scales + static_cast<int64_t>(row) * 4);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p.k_scales + static_cast<int64_t>(row) * 2);
      w[1] = *reinterpret_cast<const uint16_t*>(p.v_scales + static_cast<int64_t>(row) * 2);
    }
  }
  const uint32_t gone = __ballot_sync(0xFFFFFFFFu, miss);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, largest_byte(w[x]));
    if (lane == 0) tops[x][warp] = top;
  }
  const uint32_t low = __reduce_min_sync(0xFFFFFFFFu, row >= 0 ? largest_byte(w[1]) : 255u);
  if (lane == 0) lows[warp] = low;
  if (lane == 0) lost[warp] = (gone & 0xFFFFu ? 1u : 0u) | (gone >> 16 ? 2u : 0u);
  __syncthreads();
  const int64_t at = (static_cast<int64_t>(seq) * p.kv_heads + head) * wp.max_tiles + t;
  int c[2];
  bool uneven = false;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const uint32_t top = max(max(tops[x][0], tops[x][1]), max(tops[x][2], tops[x][3]));
    c[x] = x == 0 ? max(static_cast<int>(top) - 127 - 7, -100) : attn_value_exponent(top);
    int c_own = c[x];
    if (x == 1) {
      uneven = attn_uneven(top, min(min(lows[0], lows[1]), min(lows[2], lows[3])));
      const int less = uneven ? attn_less(c_own, largest_byte(w[x])) : 0;
      c_own -= less;
      wp.info[at].less[tid] = static_cast<uint8_t>(less);
    }
#pragma unroll
    for (int h = 0; h < BL / 2; ++h) {
      const uint32_t f = f16_pow2x2(__byte_perm(w[x], 0u, h == 0 ? 0x4140 : 0x4342), c_own + 127);
      *reinterpret_cast<uint32_t*>(&factors[x][tid * BL + 2 * h]) = row >= 0 ? f : 0u;
    }
  }
  if (tid == 0) {
    const uint32_t all = lost[0] | lost[1] << 2 | lost[2] << 4 | lost[3] << 6;
    wp.info[at].ck = c[0];
    wp.info[at].cv = c[1];
    wp.info[at].missing = all;
    wp.info[at].uneven = uneven;
    if (all != 0) atomicOr(&g_device_error, kErrorIndex);
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const uint8_t* codes = v == 0 ? k_codes : v_codes;
    uint8_t* dst = wp.tiles + (at * 2 + v) * Cfg::kF16Bytes;
#pragma unroll 4
    for (int i = 0; i < kChunks; ++i) {
      const int n = i * 128 + tid, r = n / kChunks, ch = n % kChunks;
      uint4 q = make_uint4(0u, 0u, 0u, 0u);   // a token that is not there is zero, whatever stands on its page
      if (rows[r] >= 0) q = *reinterpret_cast<const uint4*>(codes + static_cast<int64_t>(rows[r]) * D + ch * 16);
      const uint32_t f = factors[v][r * BL + (ch >> 1)] * 0x10001u;
      uint8_t* line = dst + (ch >> 2) * Cfg::kHalfTile + r * 128;
      const int p0 = (ch & 3) * 2;
      *reinterpret_cast<uint4*>(line + ((p0 ^ (r & 7)) << 4)) = make_uint4(hmul2(e4m3x2_to_f16x2(q.x), f), hmul2(e4m3x2_to_f16x2_high(q.x), f),
                                                                         hmul2(e4m3x2_to_f16x2(q.y), f), hmul2(e4m3x2_to_f16x2_high(q.y), f));
      *reinterpret_cast<uint4*>(line + (((p0 + 1) ^ (r & 7)) << 4)) = make_uint4(hmul2(e4m3x2_to_f16x2(q.z), f), hmul2(e4m3x2_to_f16x2_high(q.z), f),
                                                                               hmul2(e4m3x2_to_f16x2(q.w), f), hmul2(e4m3x2_to_f16x2_high(q.w), f));
    }
  }
}

// Adds the parts of each unit up, in the order of the tokens.  CTA (unit, eight of its rows): one warp per row.
template <int D>
__global__ void __launch_bounds__(256) attention_wide_join_kernel(const __grid_constant__ AttnWideParams wp) {
  constexpr int V = D / 32, kBatch = 4;
  const AttnParams& p = wp.a;
  const int lane = threadIdx.x & 31, unit = blockIdx.x, row = blockIdx.y * 8 + (threadIdx.x >> 5);
  grid_launch_dependents();
  grid_dependency_wait();
  const AttnWidePlan plan = *wp.plan;
  if (plan.splits <= 1 || unit >= plan.units) return;
  const AttnJoin u = p.join[unit];
  if (row >= u.n_rows) return;
  float2 total = make_float2(kAtNone, 0.0f);
  float acc[V];
#pragma unroll
  for (int e = 0; e < V; ++e) acc[e] = 0.0f;
  for (int i0 = 0; i0 < u.parts; i0 += kBatch) {
    float2 ml[kBatch];
    float v[kBatch][V];
    float top = total.x;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      ml[k] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int e = 0; e < V; ++e) v[k][e] = 0.0f;
      if (i0 + k < u.parts) {
        const int64_t at = (static_cast<int64_t>(unit) * plan.splits + i0 + k) * kWdRows + row;
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
      const float f = ex2(ml[k].x - top);
      total.y = fmaf(ml[k].y, f, total.y);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = fmaf(v[k][e], f, acc[e]);
    }
  }
  const int64_t token = u.q0 + (u.row0 + row) / p.group;
  const int qh = u.head * p.group + (u.row0 + row) % p.group;
  const float inv = total.y > 0.0f ? 1.0f / total.y : 0.0f;
#pragma unroll
  for (int e = 0; e < V; e += 2) store_attn_row(p, token, qh, D, lane * V + e, acc[e] * inv, acc[e + 1] * inv);
  if (lane == 0 && p.lse != nullptr) p.lse[token * p.q_heads + qh] = total.y > 0.0f ? (total.x + log2f(total.y)) * 0.69314718055994531f : -INFINITY;
}

}  // namespace batq
