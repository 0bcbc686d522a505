// The paged 8-bit KV cache: writing keys and values into it, and the causal
// attention that reads it (device code and launchers, included by
// kernels_attn.hip).
//
// Keys [n_blocks][Hkv][T][D] and values [n_blocks][Hkv][D][T] are e4m3 codes; a
// block of T tokens and a head share one power-of-two scale 2^(s - 127) for its
// keys and one for its values.  A power of two keeps the three fraction bits
// of every code whatever the scale (an e4m3 code is a floating number: another
// factor would buy nothing), makes a code times its scale exact in bf16, and
// makes a rescaled code exact as long as it stays normal.
#pragma once

#include "ssd_internal.h"

namespace ssd {

// Smallest s >= 1 with amax <= 448 * 2^(s - 127) (448, the largest e4m3 value, is
// 1.75 * 2^8; the biased exponent of amax less 8, one more where its fraction exceeds 0.75).
__device__ __forceinline__ int kvq_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return e < 1 ? 1 : e;
}
// 2^x, -126 <= x <= 127
__device__ __forceinline__ float kvq_pow2(int x) { return __uint_as_float((uint32_t)(x + 127) << 23); }

// what the scale has to cover: finite magnitudes
__device__ __forceinline__ float kvq_mag(float x) {
  const float m = fabsf(x);
  return m < INFINITY ? m : 0.f;
}
// x times a power of two, ready to be rounded: infinities end at the largest
// code, and a NaN is stored as zero (one would otherwise reach every later
// query of its request, through a weight of zero too)
__device__ __forceinline__ float kvq_fit(float x, float inv) {
  const float y = fminf(fmaxf(x * inv, -448.f), 448.f);
  return x == x ? y : 0.f;
}
// four codes, nearest with ties to even
__device__ __forceinline__ uint32_t kvq_code4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
typedef float kvq_f2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void kvq_value4(uint32_t codes, float (&v)[4]) {
  const kvq_f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  v[0] = lo[0], v[1] = lo[1], v[2] = hi[0], v[3] = hi[1];
}

// ---------------- writing ----------------
// Row r of the new keys and values goes to slot slots[r] (block * T + offset);
// negative and too large slots are skipped.  A wave owns one run: the rows of
// one block, consecutive rows with consecutive slots.  It starts at a row
// whose predecessor is not the slot before it, or at a block's first slot; the
// other rows' waves end at once.  The wave finds the run's largest magnitude,
// sets the scale, rewrites the block's older codes where the scale grew, and
// stores the run (which it reads a second time, from the caches).
template <typename E>
__device__ __forceinline__ float kvq_ld(const E* p);
template <>
__device__ __forceinline__ float kvq_ld<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float kvq_ld<uint16_t>(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

template <typename E>
__global__ __launch_bounds__(256) void kvq_append_kernel(KvqAppendArgs a) {
  const int lane = threadIdx.x & 63;
  const long long task = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int which = (int)(task & 1), h = (int)((task >> 1) % a.Hkv);
  const long long row = (task >> 1) / a.Hkv;
  if (row >= a.n_rows) return;
  const int T = a.T, D = a.D, cap = a.n_blocks * T;
  const int slot = a.slots[row];
  if (slot < 0 || slot >= cap) return;
  const int off = slot % T, page = slot / T;
  if (row > 0 && off != 0 && a.slots[row - 1] == slot - 1) return;
  // length of the run
  int n = 0;
  while (true) {
    const bool in = row + n + lane < a.n_rows && off + n + lane < T && a.slots[row + n + lane] == slot + n + lane;
    const uint64_t m = ~__ballot(in);
    if (m) {
      n += __builtin_ctzll(m);
      break;
    }
    n += 64;
  }
  const E* src = (const E*)(which ? a.v : a.k) + (size_t)row * (which ? a.ld_v : a.ld_k) + (size_t)h * D;
  const size_t ld = which ? a.ld_v : a.ld_k;
  uint8_t* blk = (which ? a.vc : a.kc) + ((size_t)page * a.Hkv + h) * ((size_t)T * D);
  uint8_t* ep = (which ? a.ve : a.ke) + (size_t)page * a.Hkv + h;
  float amax = 0.f;
  for (int i = lane; i < n * D; i += 64) amax = fmaxf(amax, kvq_mag(kvq_ld(src + (size_t)(i / D) * ld + i % D)));
  for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  int s = kvq_exponent(amax);
  if (off > 0) {
    const int old = *ep;
    if (old >= s) {
      s = old;
    } else {
      // 2^(old - s): a factor below every code's smallest part leaves zero
      const float f = old - s < -126 ? 0.f : kvq_pow2(old - s);
      for (int i = lane; i < off * D; i += 64) {
        uint8_t* p = which ? blk + (size_t)(i / off) * T + i % off : blk + i;
        const float x = __builtin_amdgcn_cvt_f32_fp8((int)*p, 0) * f;
        *p = (uint8_t)kvq_code4(x, x, x, x);
      }
    }
  }
  if (lane == 0) *ep = (uint8_t)s;
  const float inv = kvq_pow2(127 - s);
  for (int i = lane; i < n * D; i += 64) {
    const int t = i / D, d = i % D;
    const float x = kvq_fit(kvq_ld(src + (size_t)t * ld + d), inv);
    (which ? blk + (size_t)d * T + off + t : blk + (size_t)(off + t) * D + d)[0] = (uint8_t)kvq_code4(x, x, x, x);
  }
}

void kvq_append(const KvqAppendArgs& a, hipStream_t st) {
  const long long tasks = (long long)a.n_rows * a.Hkv * 2;
  const dim3 grid((unsigned)((tasks + 3) / 4));
  if (a.bf16) hipLaunchKernelGGL(kvq_append_kernel<uint16_t>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(kvq_append_kernel<float>, grid, dim3(256), 0, st, a);
}

// ---------------- attention ----------------
// Request b has rows cu[b] .. cu[b + 1] - 1 of q, its newest positions: row i of
// n sits at position len - n + i and sees the keys at [0, that position].  A
// position whose table entry is no block of the cache is seen by none; a row
// that sees nothing gets zeros.
//
// Plain kernel: a workgroup for each row and query head, a running maximum and
// sum over tiles of 256 keys; a thread scores one key, then sums one dim over
// its share of the tile.
template <typename E>
__global__ __launch_bounds__(256) void kvq_attn_kernel(KvqAttnArgs a) {
  __shared__ float qs[128], ps[256], red[4], part[256];
  const int tid = threadIdx.x, b = blockIdx.x / a.max_q, i = blockIdx.x - b * a.max_q, hq = blockIdx.y;
  const int D = a.D, T = a.T, h = hq / (a.Hq / a.Hkv);
  const int r0 = a.cu[b];
  const long long n = (long long)a.cu[b + 1] - r0, row = (long long)r0 + i;
  if (i >= n || row < 0 || row >= a.n_rows) return;
  const int seen = (int)min((long long)a.width * T, (long long)a.lens[b] - n + i + 1);  // keys of this row (none: <= 0)
  if (tid < D) qs[tid] = kvq_ld((const E*)a.q + row * a.ld_q + (size_t)hq * D + tid);
  const int d = tid % D, np = 256 / D, pt = tid / D;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int j0 = 0; j0 < seen; j0 += 256) {
    __syncthreads();
    const int j = j0 + tid;
    float s = -INFINITY;
    if (j < seen) {
      const int page = a.table[(size_t)b * a.width + j / T];
      if (page >= 0 && page < a.n_blocks) {
        const uint32_t* kp = (const uint32_t*)(a.kc + (((size_t)page * a.Hkv + h) * T + j % T) * D);
        float x = 0.f;
        for (int c = 0; c < D / 4; ++c) {
          float v[4];
          kvq_value4(kp[c], v);
          for (int e = 0; e < 4; ++e) x = fmaf(v[e], qs[c * 4 + e], x);
        }
        s = x * kvq_pow2((int)a.ke[(size_t)page * a.Hkv + h] - 127) * a.scale;
      }
    }
    float mt = s;
    for (int o = 32; o > 0; o >>= 1) mt = fmaxf(mt, __shfl_xor(mt, o));
    if ((tid & 63) == 0) red[tid >> 6] = mt;
    __syncthreads();
    mt = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float f = m == mt ? 1.f : expf(m - mt);  // (nothing seen so far: exp(-inf) = 0)
    const float p = s == -INFINITY ? 0.f : expf(s - mt);
    m = mt;
    ps[tid] = p;
    float lt = p;
    for (int o = 32; o > 0; o >>= 1) lt += __shfl_xor(lt, o);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = lt;
    __syncthreads();
    l = l * f + ((red[0] + red[1]) + (red[2] + red[3]));
    acc *= f;
    for (int t = pt; t < 256 && j0 + t < seen; t += np) {
      const int page = a.table[(size_t)b * a.width + (j0 + t) / T];
      if (page < 0 || page >= a.n_blocks) continue;
      const size_t head = (size_t)page * a.Hkv + h;
      const float v = __builtin_amdgcn_cvt_f32_fp8((int)a.vc[(head * D + d) * T + (j0 + t) % T], 0);
      acc = fmaf(ps[t], v * kvq_pow2((int)a.ve[head] - 127), acc);
    }
  }
  part[tid] = acc;
  __syncthreads();
  if (tid < D) {
    for (int t = 1; t < np; ++t) acc += part[t * D + tid];
    const float o = l > 0.f ? acc / l : 0.f;
    E* dst = (E*)a.o + row * a.ld_o + (size_t)hq * D + tid;
    if constexpr (sizeof(E) == 2) *dst = f2bf(o);
    else *dst = o;
  }
}

size_t kvq_attn_workspace(const KvqAttnArgs&) { return 0; }

void kvq_attention(const KvqAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.B * a.max_q), a.Hq);
  if (a.bf16) hipLaunchKernelGGL(kvq_attn_kernel<uint16_t>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(kvq_attn_kernel<float>, grid, dim3(256), 0, st, a);
}

}  // namespace ssd
