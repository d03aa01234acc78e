// New tokens into the 8-bit key/value cache: position rotation, block transform, clip, MXFP8, paged store.
//
// Per (token, head) row of head_dim channels: rotation of the first rot_dim channels (channel i with i + rot_dim / 2),
// then per 32-channel block V~ = L^T V R (x P_j, Eq. 1-2 and Algorithm 1), clip to [c_lo*min, c_hi*max] (Eq. 3-4) and
// MXFP8 (Sec. 2: E4M3, e = floor(log2 amax) - 8, saturating) for keys and values; the queries of the same tokens take
// the rotation and their own transform (the keys' dual P^-T) and are rounded once, to bf16.
//
// One thread takes one block of one row.  A CTA takes the 32 KB (256 blocks) that 256 threads hold: all rows of one
// role (queries, keys or values), so that a thread's block index, and with it its factors, never changes.  The rows
// go through shared memory because a rotation reads its partner channels, which are another thread's.
#pragma once
#include <cuda_fp16.h>

#include "ptx.cuh"
#include "quantize_act.cuh"
#include "quantize_act_tc.cuh"

namespace batq {

constexpr int kKvThreads = 256;

struct KvRole {            // queries, keys or values of a call
  const uint16_t* x;       // bf16 bits: row (token, head) at token * ld + head * head_dim
  int64_t ld;
  int32_t heads;
  int32_t tiles;           // CTAs of this role
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

// GC: size of the right factor, gr * gc == 32 (0: no role of this launch has a transform).
template <int D, int GC>
__global__ void __launch_bounds__(kKvThreads) kv_append_kernel(const __grid_constant__ KvAppendParams p) {
  constexpr int BPR = D / 32, ROWS = kKvThreads / BPR, CPR = D / 8;   // blocks, 16-byte chunks per row
  constexpr int gc = GC ? GC : 1, gr = 32 / gc;
  __shared__ __align__(16) uint4 tile[ROWS * CPR];
  grid_launch_dependents();
  int which = 0, t = static_cast<int>(blockIdx.x);
  while (which < 2 && t >= p.role[which].tiles) t -= p.role[which++].tiles;
  const KvRole& r = p.role[which];
  const int tid = threadIdx.x;
  const int64_t row0 = static_cast<int64_t>(t) * ROWS, n_rows = p.tokens * r.heads;
  // x, slots and positions may come from the grid in front
  grid_dependency_wait();
  // chunk i of block b sits at b * 4 + (i ^ ((row * BPR + b) / 2) % 4): eight neighbouring threads reading the same i
  // meet eight different groups of banks
#pragma unroll
  for (int i = 0; i < CPR * ROWS / kKvThreads; ++i) {
    const int c = i * kKvThreads + tid, lr = c / CPR, ch = c % CPR;
    const int64_t row = row0 + lr;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (row < n_rows) {
      const int64_t token = row / r.heads;
      v = ld_global_ordered_v4(r.x + token * r.ld + (row - token * r.heads) * D + ch * 8);
    }
    const int b = ch >> 2;
    tile[lr * CPR + b * 4 + ((ch & 3) ^ (((lr * BPR + b) >> 1) & 3))] = v;
  }
  __syncthreads();
  const int lr = tid / BPR, j = tid % BPR;
  const int64_t row = row0 + lr;
  if (row >= n_rows) return;
  const int64_t token = row / r.heads;
  const int head = static_cast<int>(row - token * r.heads);
  const int64_t slot = *reinterpret_cast<const volatile int64_t*>(p.slots + token);
  if (slot < 0) return;
  int64_t pos = p.rope == nullptr ? 0 : p.positions != nullptr ? *reinterpret_cast<const volatile int32_t*>(p.positions + token) : token;
  if (slot >= p.n_slots || (p.rope != nullptr && (pos < 0 || pos >= p.rope_rows))) {
    atomicOr(&g_device_error, kErrorIndex);
    return;
  }
  auto chunk = [&](int ch) {
    const int b = ch >> 2;
    return tile[lr * CPR + b * 4 + ((ch & 3) ^ (((lr * BPR + b) >> 1) & 3))];
  };
  float o[32];
  const float* table = p.rope + pos * p.rot_dim;
  const int half = p.rot_dim >> 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int ch = j * 4 + i;
    float x[8];
    unpack_bf16x8(chunk(ch), x);
    if (r.rotate && ch * 8 < p.rot_dim) {
      const bool upper = ch * 8 >= half;
      const int f = upper ? ch * 8 - half : ch * 8;
      float y[8];
      unpack_bf16x8(chunk((upper ? f : f + half) >> 3), y);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 c = __ldg(reinterpret_cast<const float4*>(table + f) + h);
        const float4 s = __ldg(reinterpret_cast<const float4*>(table + half + f) + h);
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[8 * i + 4 * h + e] = fmaf(x[4 * h + e], cs[e], upper ? y[4 * h + e] * sn[e] : -y[4 * h + e] * sn[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) o[8 * i + e] = x[e];
    }
  }
  if (GC != 0 && r.xform) {
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
    return;
  }
  float mn = o[0], mx = o[0];
#pragma unroll
  for (int i = 1; i < 32; ++i) {
    mn = fminf(mn, o[i]);
    mx = fmaxf(mx, o[i]);
  }
  if (r.clip_lo != nullptr) {
    const float lo = __ldg(r.clip_lo + j) * mn, hi = __ldg(r.clip_hi + j) * mx;
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = fminf(fmaxf(o[i], lo), hi);
    const float a = fminf(fmaxf(mn, lo), hi), b = fminf(fmaxf(mx, lo), hi);
    mn = a; mx = b;
  }
  const float amax = fmaxf(fabsf(mn), fabsf(mx));
  const int sbyte = max(static_cast<int>(__float_as_uint(amax) >> 23) - 8, 0);
  const float inv = __uint_as_float(static_cast<uint32_t>(254 - sbyte) << 23);
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = e4m3x4_pack(o[4 * i] * inv, o[4 * i + 1] * inv, o[4 * i + 2] * inv, o[4 * i + 3] * inv);
  const int64_t page = slot >> p.page_shift, off = slot & ((int64_t(1) << p.page_shift) - 1);
  const int64_t at = (((page * r.heads + head) << p.page_shift) + off) * BPR + j;   // in blocks
  uint4* dst = reinterpret_cast<uint4*>(r.codes + at * 32);
  dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
  dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
  r.scales[at] = static_cast<uint8_t>(sbyte);
}

}  // namespace batq
