// Small device functions of the kernels that read the 8-bit committed cache.
#pragma once

#include <cuda.h>
#include <cuda_fp8.h>

#include "cod_internal.cuh"

struct Kv8Params {
  const __nv_bfloat16 *q, *kb, *vb;          // [S][W][n_q|n_kv][hd]; q and k_blk rotated by the kernels if inv_freq is given
  const uint8_t* pool;
  const float* scale;
  const __nv_bfloat16* carry;
  const int *block_table, *committed_len, *carry_len;
  const double* inv_freq;
  int use_carry, layer, S, W, rep, n_kv, n_pages, max_pages, max_batch, cap;
  int unit, setup;                           // work line: pages per unit; what it costs to begin a segment, in units
  int line_blocks;                           // how many stretches the work line is cut into
  int run_ahead;                             // finish kernel: what it reads before its wait is older than the paged kernel
  float *part_o, *part_ml;                   // [slot][M][hd], [slot][M][4]: d, r, l, l_carry (the sums are relative to r, o to r + d)
  uint32_t* status;
};

namespace kv8 {

constexpr int PAGE = 16;              // tokens per page and scale block

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {      // the low 16 bits; exact
  uint32_t d;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"(static_cast<unsigned short>(two)));
  return d;
}
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(four));
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t two) {
  const uint32_t h = e4m3x2_to_f16x2(two);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// loads that are issued where they stand (an ordinary one may be moved down to its first use)
__device__ __forceinline__ int ld_now(const int* p) {
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ float2 ld_now(const float2* p) {
  float2 v;
  asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ float4 ld_now(const float4* p) {
  float4 v;
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}
// the pages' copies: read once (by both row groups of a block of more than 64 rows at about the same time), they leave L2 first
__device__ __forceinline__ uint64_t l2_evict_first() {
  uint64_t pol;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
  return pol;
}
// one box of pages
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, int row, uint32_t bar, uint64_t pol) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(bar), "l"(pol) : "memory");
}
// N words from global memory (8 or 16 bytes, aligned to their size)
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  } else {
    const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
    w[0] = u.x; w[1] = u.y;
  }
}
// N bf16 elements (8 or 16) as floats
template <int N>
__device__ __forceinline__ void load_chunk(const __nv_bfloat16* p, float (&v)[N]) {
#pragma unroll
  for (int k = 0; k < N; k += 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p + k);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[k + 2 * e] = __uint_as_float(w[e] << 16); v[k + 2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u); }
  }
}
// N e4m3 bytes (8 or 16) times their page's scale
template <int N>
__device__ __forceinline__ void load_bytes(const uint8_t* p, float f, float (&v)[N]) {
  uint32_t w[N / 4];
  load_words<N / 4>(p, w);
#pragma unroll
  for (int e = 0; e < N / 4; ++e) {
    const float2 lo = e4m3x2_to_float2(w[e] & 0xFFFFu), hi = e4m3x2_to_float2(w[e] >> 16);
    v[4 * e] = lo.x * f; v[4 * e + 1] = lo.y * f; v[4 * e + 2] = hi.x * f; v[4 * e + 3] = hi.y * f;
  }
}
// rotary embedding of element pairs (lo[k], hi[k]); cs: their cosines, cs + half: their sines
template <int N>
__device__ __forceinline__ void rotate_chunk(float (&lo)[N], float (&hi)[N], const float* cs, int half) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float a = lo[k], b = hi[k], c = cs[k], s = cs[half + k];
    lo[k] = a * c - b * s;
    hi[k] = b * c + a * s;
  }
}

// ---------------------------------------------------------------------------- the work line
// The whole pages of all (sequence, KV head) pairs, in units of `unit` pages (a pair's last unit may hold fewer), lie one
// behind the other, each pair behind `setup` empty units that stand for the cost of beginning it; block i of n takes units
// [i per, (i + 1) per).
constexpr int MIN_PER = 16;            // shortest stretch, in pages
struct Stretch { int w0, w1, s, base; };                     // [w0, w1); the sequence that holds w0, and where it begins
struct Segment { int s, h, L, u0, u1, base, w; bool any; };  // units [u0, u1) of one pair; w: where the next one begins

__device__ __forceinline__ int clamped_len(const Kv8Params& p, int s) { return max(0, min(p.committed_len[s], p.max_pages * PAGE)); }
__device__ __forceinline__ int units_of(const Kv8Params& p, int L, int unit) {           // of one pair, its setup included
  return L < PAGE ? 0 : p.setup + (L / PAGE + unit - 1) / unit;
}

// units per block, from the line's length
__device__ __forceinline__ int units_per(int total, int blocks, int unit) { return max((total + blocks - 1) / blocks, (MIN_PER + unit - 1) / unit); }
// Where sequence s begins on the line, and the units per block. Every thread of the block's N warps takes part; sh: 2 N ints.
template <int N>
__device__ __forceinline__ void place_of(const Kv8Params& p, int s, int* sh, int& base, int& per) {
  int before = 0, total = 0;
  for (int i = threadIdx.x; i < p.S; i += N * 32) {
    const int v = p.n_kv * units_of(p, clamped_len(p, i), p.unit);
    total += v;
    if (i < s) before += v;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  total = __reduce_add_sync(0xffffffffu, total);
  if ((threadIdx.x & 31) == 0) { sh[threadIdx.x >> 5] = before; sh[N + (threadIdx.x >> 5)] = total; }
  __syncthreads();
  base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < N; ++w) { base += sh[w]; total += sh[N + w]; }
  per = units_per(total, p.line_blocks, p.unit);
}
// exclusive prefix sum over the block's threads (N warps) and its total; red: N ints
template <int N>
__device__ __forceinline__ int block_prefix(int v, int* red, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                           // red may still be read from the call before
  if (lane == 31) red[warp] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < N; ++w) {
    if (w < warp) before += red[w];
    total += red[w];
  }
  return before + x - v;
}
// This block's stretch; every thread of the block's N warps takes part (the barriers inside also publish what was set up
// before). sh: N + 2 ints of shared memory. `chief` reports bad lengths. False: nothing to do.
template <int N>
__device__ __forceinline__ bool cut_line(const Kv8Params& p, int unit, int i, int n, bool chief, int* sh, Stretch& out, uint32_t& flags) {
  int total = 0;
  for (int s0 = 0; s0 < p.S; s0 += N * 32) {
    const int s = s0 + threadIdx.x;
    int part;
    block_prefix<N>(s < p.S ? p.n_kv * units_of(p, clamped_len(p, s), unit) : 0, sh, part);
    total += part;
  }
  const int per = units_per(total, n, unit);
  const bool some = static_cast<long long>(i) * per < total;
  if (!some && !chief) return false;
  out.w0 = i * per;
  out.w1 = min(total - out.w0, per) + out.w0;
  int before = 0;
  for (int s0 = 0; s0 < p.S; s0 += N * 32) {
    const int s = s0 + threadIdx.x;
    const int v = s < p.S ? p.n_kv * units_of(p, clamped_len(p, s), unit) : 0;
    int all;
    const int base = before + block_prefix<N>(v, sh, all);
    before += all;
    if (s < p.S && base <= out.w0 && out.w0 < base + v) { sh[N] = s; sh[N + 1] = base; }
    if (chief && s < p.S && (p.committed_len[s] < 0 || p.committed_len[s] > p.max_pages * PAGE)) flags |= COD_DEV_BAD_LEN;
  }
  if (!some) {                               // no whole page anywhere
    if (flags) atomicOr(p.status, flags);
    return false;
  }
  __syncthreads();
  out.s = sh[N];
  out.base = sh[N + 1];
  return true;
}
__device__ __forceinline__ void next_segment(const Kv8Params& p, const Stretch& line, int unit, Segment& k) {
  for (;;) {
    k.any = k.w < line.w1;
    if (!k.any) return;
    const int units = units_of(p, k.L, unit), end = k.base + p.n_kv * units;
    if (k.w >= end) {                        // the next sequence
      k.base = end;
      ++k.s;
      k.L = clamped_len(p, k.s);
      continue;
    }
    const int in = k.w - k.base;
    k.h = in / units;
    const int at = in - k.h * units, to = min(units, line.w1 - k.w + at);
    k.w += to - at;
    k.u0 = max(at - p.setup, 0);
    k.u1 = to - p.setup;
    if (k.u0 < k.u1) return;                 // else: the stretch ends in the pair's setup
  }
}
__device__ __forceinline__ Segment first_segment(const Kv8Params& p, const Stretch& line, int unit) {
  Segment k;
  k.s = line.s; k.base = line.base; k.w = line.w0; k.L = clamped_len(p, k.s);
  k.h = 0; k.u0 = 0; k.u1 = 0;
  next_segment(p, line, unit, k);
  return k;
}

}  // namespace kv8
