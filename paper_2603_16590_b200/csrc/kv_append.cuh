// New tokens into the 8-bit key/value cache: position rotation, block transform, clip, MXFP8, paged store.
//
// Per (token, head) row of head_dim channels: rotation of the first rot_dim channels (channel i with i + rot_dim / 2),
// then per 32-channel block V~ = L^T V R (x P_j, Eq. 1-2 and Algorithm 1), clip to [c_lo*min, c_hi*max] (Eq. 3-4) and
// MXFP8 (Sec. 2: E4M3, e = floor(log2 amax) - 8, saturating) for keys and values; the queries of the same tokens take
// the rotation and their own transform (the keys' dual P^-T) and are rounded once, to bf16.
//
// One thread takes one block of one row.  A CTA takes tiles of 256 blocks, whole rows of one role (queries, keys or
// values), so that a thread's block index never changes and the factors of a head's blocks are put into shared memory once.
// The rows go through shared memory, the next tile's on their way while this one is worked on, because a rotation reads its
// partner channels, which are another thread's.
//
// Bound by instructions before it is by memory (3.1 bytes a key or value element): the 4 x 8 form therefore runs on packed
// fp32 pairs, 224 instructions per block instead of 384:
//   W = L^T V    pairs of neighbouring columns, the entries of L twice in a word pair;
//   W R          pairs of neighbouring terms of the sum, R's columns stored in such pairs; their halves are added last.
#pragma once
#include <cuda_fp16.h>

#include "ptx.cuh"
#include "quantize_act.cuh"
#include "quantize_act_tc.cuh"
#include "quantize_act_warp.cuh"

namespace batq {

constexpr int kKvThreads = 256;

struct KvRole {            // queries, keys or values of a call
  const uint16_t* x;       // bf16 bits: row (token, head) at token * ld + head * head_dim
  int64_t ld;
  int32_t heads;
  uint32_t heads_inv;      // 2^32 / heads, rounded up: n / heads = n * heads_inv >> 32 for n * heads < 2^32
  int32_t head_step;       // (ctas * rows of a tile) % heads, / heads: from a CTA's tile to its next one
  int64_t token_step;
  int64_t tiles;           // tiles of this role
  int32_t ctas;            // CTAs, which share the tiles
  int32_t rotate;          // != 0: the position rotation applies
  int32_t xform;           // != 0: left / right below apply
  const float* left;
  const float* right;
  int32_t left_stride, right_stride;
  const float* clip_lo;    // [head_dim / 32] or NULL
  const float* clip_hi;
  uint8_t* codes;          // keys, values: [page][head][token of the page][head_dim]
  uint8_t* scales;         //               [page][head][token of the page][head_dim / 32]
  uint16_t* out;           // queries: bf16, row (token, head) at token * ldo + head * head_dim
  int64_t ldo;
};

struct KvAppendParams {
  KvRole role[3];
  int64_t tokens;
  const int64_t* slots;      // [tokens]; < 0: the row is padding
  int64_t n_slots;           // pages * page_size
  int32_t page_shift;        // log2 page_size
  const float* rope;         // [rope_rows][rot_dim]: cosines, then sines; NULL: no rotation
  int64_t rope_rows;
  const int32_t* positions;  // [tokens], NULL: token i has row i of the table
  int32_t rot_dim;
};

__device__ __forceinline__ void unpack_bf16x8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    v[2 * h] = __uint_as_float(w[h] << 16);
    v[2 * h + 1] = __uint_as_float(w[h] & 0xFFFF0000u);
  }
}

// The same in pairs of neighbours.
__device__ __forceinline__ void unpack_bf16x8_pairs(const uint4& q, uint64_t (&v)[4]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int h = 0; h < 4; ++h) v[h] = f32x2_pack(__uint_as_float(w[h] << 16), __uint_as_float(w[h] & 0xFFFF0000u));
}
// x cos + y sin of eight channels (y: the partners, negated in the first half of a head).
__device__ __forceinline__ void rotate_pairs(const uint64_t (&x)[4], const uint64_t (&y)[4], const float* cos, const float* sin, uint64_t* out) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const ulonglong2 c = __ldg(reinterpret_cast<const ulonglong2*>(cos) + h), s = __ldg(reinterpret_cast<const ulonglong2*>(sin) + h);
    out[2 * h] = f32x2_fma(x[2 * h], c.x, f32x2_mul(y[2 * h], s.x));
    out[2 * h + 1] = f32x2_fma(x[2 * h + 1], c.y, f32x2_mul(y[2 * h + 1], s.y));
  }
}

// 16 bytes global -> shared, the rest behind `bytes` as zeros; waiting for all but the newest N groups of the thread's.
__device__ __forceinline__ void cp_async_16(uint32_t dst_smem, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst_smem), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// GC: size of the right factor, gr * gc == 32 (0: no role of this launch has a transform).
template <int D, int GC>
__global__ void __launch_bounds__(kKvThreads, GC == 8 || GC == 0 ? 3 : 2) kv_append_kernel(const __grid_constant__ KvAppendParams p) {
  constexpr int BPR = D / 32, ROWS = kKvThreads / BPR, CPR = D / 8;   // blocks, 16-byte chunks per row
  constexpr int gc = GC ? GC : 1, gr = 32 / gc;
  constexpr int kFactorStride = 100;   // words of a block's factors: 32 pairs of R, 16 pairs of L, and 4 so that blocks meet in no bank
  __shared__ __align__(16) uint4 tiles[2][ROWS * CPR];
  __shared__ __align__(16) float factors[GC == 8 ? BPR * kFactorStride : 1];
  grid_launch_dependents();
  int which = 0, cta = static_cast<int>(blockIdx.x);
  while (which < 2 && cta >= p.role[which].ctas) cta -= p.role[which++].ctas;
  const KvRole& r = p.role[which];
  const int tid = threadIdx.x, lr = tid / BPR, j = tid % BPR;
  const bool xform = GC != 0 && r.xform != 0;
  if (GC == 8 && xform)
    for (int i = tid; i < BPR * 48; i += kKvThreads) {
      const int b = i / 48, k = i % 48;
      float x, y;
      if (k < 32) {   // pair k: rows 2 (k / 8), + 1 of column k % 8 of R
        const float* R = r.right + static_cast<int64_t>(b) * r.right_stride + (k >> 3) * 16 + (k & 7);
        x = __ldg(R);
        y = __ldg(R + 8);
      } else {        // entry k - 32 of L, twice
        x = y = __ldg(r.left + static_cast<int64_t>(b) * r.left_stride + k - 32);
      }
      *reinterpret_cast<float2*>(factors + b * kFactorStride + 2 * k) = make_float2(x, y);
    }
  const float clip_lo = r.clip_lo != nullptr ? __ldg(r.clip_lo + j) : 1.0f, clip_hi = r.clip_lo != nullptr ? __ldg(r.clip_hi + j) : 1.0f;
  const int64_t n_rows = p.tokens * r.heads;
  // x, slots and positions may come from the grid in front
  grid_dependency_wait();
  // chunk i of block b sits at b * 4 + (i ^ ((row * BPR + b) / 2) % 4): eight neighbouring threads reading the same i
  // meet eight different groups of banks
  auto place = [](int row, int ch) {
    const int b = ch >> 2;
    return row * CPR + b * 4 + ((ch & 3) ^ (((row * BPR + b) >> 1) & 3));
  };
  auto token_of = [&](int64_t token0, int n, int& head) {   // n heads on from head 0 of token0
    const int t = r.heads == 1 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), r.heads_inv));
    head = n - t * r.heads;
    return token0 + t;
  };
  // rows of a tile from head `head0` of token `token0` on; fetched by all threads, always the same chunk of a row
  const int fetch_row = tid / CPR, fetch_ch = tid % CPR;
  auto fetch = [&](int64_t tile, int64_t token0, int head0, int stage) {
    if (tile < r.tiles) {
      const int rows = static_cast<int>(min(static_cast<int64_t>(ROWS), n_rows - tile * ROWS));
#pragma unroll
      for (int i = 0; i < CPR * ROWS / kKvThreads; ++i) {
        const int row = i * (kKvThreads / CPR) + fetch_row;
        int head;
        const int64_t token = token_of(token0, head0 + row, head);
        const bool there = row < rows;
        cp_async_16(smem_u32(&tiles[stage][place(row, fetch_ch)]), r.x + (there ? token * r.ld + (head * D + fetch_ch * 8) : 0), there ? 16 : 0);
      }
    }
    cp_async_commit();
  };
  int64_t token0 = static_cast<int64_t>(cta) * ROWS / r.heads;
  int head0 = static_cast<int>(static_cast<int64_t>(cta) * ROWS - token0 * r.heads);
  fetch(cta, token0, head0, 0);
  int stage = 0;
  for (int64_t t = cta; t < r.tiles; t += r.ctas, stage ^= 1) {
    int head;
    const int64_t token = token_of(token0, head0 + lr, head);
    int64_t slot = -1, pos = 0;
    if (t * ROWS + lr < n_rows) {
      slot = *reinterpret_cast<const volatile int64_t*>(p.slots + token);
      if (p.rope != nullptr) pos = p.positions != nullptr ? *reinterpret_cast<const volatile int32_t*>(p.positions + token) : token;
    }
    if (slot >= p.n_slots || (slot >= 0 && p.rope != nullptr && (pos < 0 || pos >= p.rope_rows))) {   // all of the token, the values too
      atomicOr(&g_device_error, kErrorIndex);
      slot = -1;
    }
    cp_async_wait<0>();
    __syncthreads();   // the tile is here (and the factors), the other one is free
    token0 += r.token_step;
    head0 += r.head_step;
    if (head0 >= r.heads) { head0 -= r.heads; ++token0; }
    fetch(t + r.ctas, token0, head0, stage ^ 1);
    if (slot < 0) continue;   // (every thread of the CTA makes the same turns: the barrier above is met by all)
    const uint4* tile = tiles[stage];
    float o[32];
    uint64_t v[16];   // the block, pairs of channels
    if (r.rotate && p.rot_dim == D) {   // whole heads: the partner is the same chunk of the block half a head away
      const bool upper = j >= BPR / 2;
      const uint32_t sign = upper ? 0u : 0x80008000u;
      const float* cs = p.rope + pos * D + (j % (BPR / 2)) * 32;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint64_t x[4], y[4];
        unpack_bf16x8_pairs(tile[place(lr, j * 4 + i)], x);
        const uint4 w = tile[place(lr, (j ^ (BPR / 2)) * 4 + i)];
        unpack_bf16x8_pairs(make_uint4(w.x ^ sign, w.y ^ sign, w.z ^ sign, w.w ^ sign), y);
        rotate_pairs(x, y, cs + i * 8, cs + D / 2 + i * 8, v + 4 * i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = j * 4 + i, half = p.rot_dim >> 1;
        uint64_t x[4], y[4];
        unpack_bf16x8_pairs(tile[place(lr, ch)], x);
        if (r.rotate && ch * 8 < p.rot_dim) {
          const bool upper = ch * 8 >= half;
          const uint32_t sign = upper ? 0u : 0x80008000u;
          const int f = upper ? ch * 8 - half : ch * 8;
          const uint4 w = tile[place(lr, (upper ? f : f + half) >> 3)];
          unpack_bf16x8_pairs(make_uint4(w.x ^ sign, w.y ^ sign, w.z ^ sign, w.w ^ sign), y);
          rotate_pairs(x, y, p.rope + pos * p.rot_dim + f, p.rope + pos * p.rot_dim + half + f, v + 4 * i);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * i + e] = x[e];
        }
      }
    }
    if (GC != 8 || !xform) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f32x2_unpack(v[i], o[2 * i], o[2 * i + 1]);
    }
    if (GC == 8 && xform) {
      const float* fac = factors + j * kFactorStride;
      uint64_t w[4][4];   // W = L^T V, pairs of columns
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const ulonglong2 l0 = *reinterpret_cast<const ulonglong2*>(fac + 64 + i * 8), l1 = *reinterpret_cast<const ulonglong2*>(fac + 64 + i * 8 + 4);
        const uint64_t l[4] = {l0.x, l0.y, l1.x, l1.y};
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
          for (int c = 0; c < 4; ++c) w[rr][c] = i == 0 ? f32x2_mul(l[rr], v[c]) : f32x2_fma(l[rr], v[4 * i + c], w[rr][c]);
      }
#pragma unroll
      for (int c = 0; c < 8; c += 2) {   // two columns of R at a time
        uint64_t acc[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(fac + (k * 8 + c) * 2);
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) {
            acc[rr][0] = k == 0 ? f32x2_mul(w[rr][k], q.x) : f32x2_fma(w[rr][k], q.x, acc[rr][0]);
            acc[rr][1] = k == 0 ? f32x2_mul(w[rr][k], q.y) : f32x2_fma(w[rr][k], q.y, acc[rr][1]);
          }
        }
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float a, b;
            f32x2_unpack(acc[rr][h], a, b);
            o[8 * rr + c + h] = a + b;
          }
      }
    } else if (GC != 0 && xform) {
      const float* R = r.right + static_cast<int64_t>(j) * r.right_stride;
      const float* L = r.left + static_cast<int64_t>(j) * r.left_stride;
      // V R, row by row, in place
#pragma unroll
      for (int i = 0; i < gr; ++i) {
        float u[gc];
#pragma unroll
        for (int c = 0; c < gc; ++c) u[c] = 0.0f;
#pragma unroll
        for (int cc = 0; cc < gc; ++cc)
#pragma unroll
          for (int c = 0; c < gc; ++c) u[c] = fmaf(o[i * gc + cc], __ldg(R + cc * gc + c), u[c]);
#pragma unroll
        for (int c = 0; c < gc; ++c) o[i * gc + c] = u[c];
      }
      // L^T (V R), column by column
#pragma unroll
      for (int c = 0; c < gc; ++c) {
        float u[gr];
#pragma unroll
        for (int i = 0; i < gr; ++i) u[i] = 0.0f;
#pragma unroll
        for (int ii = 0; ii < gr; ++ii)
#pragma unroll
          for (int i = 0; i < gr; ++i) u[i] = fmaf(o[ii * gc + c], __ldg(L + ii * gr + i), u[i]);
#pragma unroll
        for (int i = 0; i < gr; ++i) o[i * gc + c] = u[i];
      }
    }
    if (r.out != nullptr) {
      uint4* dst = reinterpret_cast<uint4*>(r.out + token * r.ldo + static_cast<int64_t>(head) * D + j * 32);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(o[8 * i + 2 * h], o[8 * i + 2 * h + 1]);
          w[h] = *reinterpret_cast<const uint32_t*>(&b);
        }
        dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      continue;
    }
    float mn = INFINITY, mx = -INFINITY;   // NaN counts as neither
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      mn = fminf(mn, o[i]);
      mx = fmaxf(mx, o[i]);
    }
    // Without a clip the ratios are 1 and the bounds the block's own: they take a NaN to a number, to 0 where there is none
    // in the block.  No NaN code is ever stored: in an attention it would reach rows that do not see its token, as 0 times
    // NaN; and no scale that is larger than the numbers need: a tile's keys stand in f16 under one exponent there.
    {
      if (!(mn <= mx)) mn = mx = 0.0f;
      const float lo = clip_lo * mn, hi = clip_hi * mx;
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = fminf(fmaxf(o[i], lo), hi);
      const float a = fminf(fmaxf(mn, lo), hi), b = fminf(fmaxf(mx, lo), hi);
      mn = a; mx = b;
    }
    const float amax = fmaxf(fabsf(mn), fabsf(mx));
    const int sbyte = max(static_cast<int>(__float_as_uint(amax) >> 23) - 8, 0);
    const float inv = __uint_as_float(static_cast<uint32_t>(254 - sbyte) << 23);
    const uint64_t inv2 = f32x2_pack(inv, inv);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a, b, c, d;
      f32x2_unpack(f32x2_mul(f32x2_pack(o[4 * i], o[4 * i + 1]), inv2), a, b);
      f32x2_unpack(f32x2_mul(f32x2_pack(o[4 * i + 2], o[4 * i + 3]), inv2), c, d);
      w[i] = e4m3x4_pack(a, b, c, d);
    }
    const int64_t page = slot >> p.page_shift, off = slot & ((int64_t(1) << p.page_shift) - 1);
    const int64_t at = (((page * r.heads + head) << p.page_shift) + off) * BPR + j;   // in blocks
    uint4* dst = reinterpret_cast<uint4*>(r.codes + at * 32);
    dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
    dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
    r.scales[at] = static_cast<uint8_t>(sbyte);
  }
}

}  // namespace batq
