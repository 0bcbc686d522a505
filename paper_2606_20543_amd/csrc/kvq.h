// The paged 8-bit KV cache: writing keys and values into it, and the causal
// attention that reads it (device code and launchers, included by
// kernels_attn.hip).
//
// Keys [n_blocks][Hkv][T][D] and values [n_blocks][Hkv][D][T] are e4m3 codes; a
// block of T tokens and a head share one power-of-two scale 2^(s - 127) for its
// keys and one for its values.  A power of two keeps the three fraction bits
// of every code whatever the scale (an e4m3 code is a floating number: another
// factor would buy nothing), makes a code times its scale exact in bf16 (but what lies
// below 2^-133), and makes a rescaled code exact as long as it stays normal.
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
// The scale of codes on their way in: 1 / 2^(s - 127), and the largest code.  That is 448 but at s = 247, the exponent of
// magnitudes above 448 * 2^119: there codes above 240 stand for 2^128 and more, which neither fp32 nor the
// bf16 operands of the attention hold.
struct KvqScale {
  float inv, top;
  __device__ __forceinline__ explicit KvqScale(int s) : inv(kvq_pow2(127 - s)), top(s < 247 ? 448.f : 240.f) {}
};
// x under the scale, ready to be rounded: infinities end at the largest
// code, and a NaN is stored as zero (one would otherwise reach every later
// query of its request, through a weight of zero too)
__device__ __forceinline__ float kvq_fit(float x, const KvqScale& sc) {
  const float y = fminf(fmaxf(x * sc.inv, -sc.top), sc.top);
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
// negative and too large slots are skipped.  A run is the rows of one block:
// consecutive rows with consecutive slots.  It starts at a row whose
// predecessor is not the slot before it, or at a block's first slot.  A run's
// largest magnitude gives the scale; the block's older codes are rewritten where
// the scale grew, then the run is stored.
//
// Nothing is computed to speak of: the bytes bound it (8 heads of 128, 16 prompts of up to 2048
// rows after one: 134 MB, 26 us at the rate of a large copy; 41 us a call, 38 of them the
// kernel), and, for single tokens, the launch (8.1 us a call, 6.5 the kernel).  Where a window of rows starts one or
// two runs, a workgroup takes them together and holds the elements between the maximum and the
// codes, so the rows are read once; where it starts more (short runs), a wave takes each and
// reads it a second time, from the caches (every run by a wave of its own: 47 us for the prompts).
template <typename E>
__device__ __forceinline__ float kvq_ld(const E* p);
template <>
__device__ __forceinline__ float kvq_ld<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float kvq_ld<uint16_t>(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// o / l as four elements of the output, zeros where no key was seen
__device__ __forceinline__ void kvq_store4(float* p, floatx4 o, float l) {
  const float f = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) p[e] = o[e] * f;
}
__device__ __forceinline__ void kvq_store4(uint16_t* p, floatx4 o, float l) {
  const float f = l > 0.f ? 1.f / l : 0.f;
  const uint32_t x = cvt2bf(o[0] * f, o[1] * f), y = cvt2bf(o[2] * f, o[3] * f);
  p[0] = (uint16_t)x, p[1] = (uint16_t)(x >> 16), p[2] = (uint16_t)y, p[3] = (uint16_t)(y >> 16);
}

// N neighbouring elements, read by one load where ALIGNED
template <typename E, int N, bool ALIGNED>
struct alignas(ALIGNED ? sizeof(E) * N : sizeof(E)) KvqVec {
  E v[N];
};

// a run's row r, in elements
template <bool NEAR>
__device__ __forceinline__ size_t kvq_row(int r, size_t ld) {
  return NEAR ? (uint32_t)r * (uint32_t)ld : (size_t)r * ld;
}
__device__ __forceinline__ float kvq_max64(float m) {
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  return m;
}
// largest finite magnitude of n rows of D elements, in every lane: 16 bytes a lane and load where
// the rows allow it (VEC), else two elements
template <typename E, bool VEC>
__device__ __forceinline__ float kvq_amax(const E* src, size_t ld, int n, int D, int lane) {
  constexpr int N = VEC ? 16 / (int)sizeof(E) : 2, U = 4;  // U loads in flight (rows past the last: that one again)
  typedef KvqVec<E, N, VEC> V;
  const int per = D / N, step = 64 / per, c = (lane % per) * N;
  float m = 0.f;
  for (int r = lane / per; r < n; r += U * step) {
    V x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *(const V*)(src + kvq_row<VEC>(min(r + u * step, n - 1), ld) + c);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, kvq_mag(kvq_ld(&x[u].v[e])));
  }
  return kvq_max64(m);
}

// codes times f (a power of two), rounded again, where keep has ones
__device__ __forceinline__ uint32_t kvq_again(uint32_t codes, float f, uint32_t keep) {
  float v[4];
  kvq_value4(codes, v);
  return (kvq_code4(v[0] * f, v[1] * f, v[2] * f, v[3] * f) & keep) | (codes & ~keep);
}
__device__ __forceinline__ uint32_t kvq_low_bytes(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

// rows [0, n) of src to tokens off .. of a block's keys [T][D]
template <typename E, bool VEC>
__device__ __forceinline__ void kvq_put_keys(const E* src, size_t ld, int n, int D, int off, const KvqScale& sc, uint8_t* blk, int lane) {
  constexpr int N = VEC ? 16 / (int)sizeof(E) : 2, U = 4;
  typedef KvqVec<E, N, VEC> V;
  const int per = D / N, step = 64 / per, c = (lane % per) * N;
  for (int r = lane / per; r < n; r += U * step) {
    V x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *(const V*)(src + kvq_row<VEC>(min(r + u * step, n - 1), ld) + c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r + u * step >= n) break;
      uint8_t* p = blk + (size_t)(off + r + u * step) * D + c;
      float y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) y[e] = kvq_fit(kvq_ld(&x[u].v[e]), sc);
      if constexpr (N == 2) {
        *(uint16_t*)p = (uint16_t)kvq_code4(y[0], y[1], 0.f, 0.f);
      } else {
#pragma unroll
        for (int e = 0; e < N; e += 4) *(uint32_t*)(p + e) = kvq_code4(y[e], y[e + 1], y[e + 2], y[e + 3]);
      }
    }
  }
}

// tokens t0 .. t0 + 15 of a dim's row, those in [off, end)
__device__ __forceinline__ void kvq_put16(uint8_t* row, int t0, int off, int end, const float (&y)[16]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = kvq_code4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
  if (t0 >= off && t0 + 16 <= end) {
    *(uint4*)(row + t0) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (t0 + j >= off && t0 + j < end) row[t0 + j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
  }
}
// the same for values [D][T]: a lane owns two neighbouring dims and takes 16 tokens at a time, which
// are 16 bytes of a dim's row where the run covers them all
template <typename E, bool VEC>
__device__ __forceinline__ void kvq_put_values(const E* src, size_t ld, int n, int D, int T, int off, const KvqScale& sc, uint8_t* blk,
                                               int lane) {
  typedef KvqVec<E, 2, VEC> V;
  const int per = D / 2, d = (lane % per) * 2, groups = 64 / per;
  for (int t0 = (off & ~15) + 16 * (lane / per); t0 < off + n; t0 += 16 * groups) {
    V x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = *(const V*)(src + kvq_row<VEC>(min(max(t0 + j - off, 0), n - 1), ld) + d);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float y[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = kvq_fit(kvq_ld(&x[j].v[e]), sc);
      kvq_put16(blk + (size_t)(d + e) * T, t0, off, off + n, y);
    }
  }
}

// a run, for one head of the keys (which = 0) or the values
template <typename E>
struct KvqRun {
  int n, off, page;  // rows; the first one's token in its block
  const E* src;
  size_t ld;
  uint8_t *blk, *ep;
  __device__ __forceinline__ KvqRun(const KvqAppendArgs& a, int which, int h, int row, int slot, int rows) {
    const int T = a.T;
    n = rows, off = slot & (T - 1), page = slot / T;
    ld = which ? a.ld_v : a.ld_k;
    src = (const E*)(which ? a.v : a.k) + (size_t)row * ld + (size_t)h * a.D;
    blk = (which ? a.vc : a.kc) + ((size_t)page * a.Hkv + h) * ((size_t)T * a.D);
    ep = (which ? a.ve : a.ke) + (size_t)page * a.Hkv + h;
  }
  // the codes before the run, by NT threads, where the exponent grew from old to s
  template <int NT>
  __device__ __forceinline__ void rescale(int which, int T, int D, int old, int s, int t) const {
    if (off == 0 || s <= old) return;
    // 2^(old - s): a factor below every code's smallest part leaves zero
    const float f = old - s < -126 ? 0.f : kvq_pow2(old - s);
    if (which) {
      const int words = (off + 3) / 4;
      for (int i = t; i < words * D; i += NT) {
        uint32_t* p = (uint32_t*)(blk + (size_t)(i / words) * T) + i % words;
        *p = kvq_again(*p, f, kvq_low_bytes(off - 4 * (i % words)));
      }
    } else {
      for (int i = t; i < off * D / 4; i += NT) {
        uint32_t* p = (uint32_t*)blk + i;
        *p = kvq_again(*p, f, ~0u);
      }
    }
  }
};
// The exponent for a workgroup's elements (m: a thread's largest), set; returns the codes' scale.
template <typename E>
__device__ __forceinline__ KvqScale kvq_shared_scale(const KvqRun<E>& run, int which, int T, int D, float m, uint32_t* red) {
  m = kvq_max64(m);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[wave] = __float_as_uint(m);
    if (wave == 0) red[4] = run.off > 0 ? *run.ep : 0;
  }
  __syncthreads();
  const uint32_t top = max(max(red[0], red[1]), max(red[2], red[3]));  // of magnitudes: ordered like their bits
  const int old = (int)red[4], s = max(kvq_exponent(__uint_as_float(top)), old);
  if (run.off > 0 && s > old) {  // (the same in the whole workgroup)
    run.template rescale<256>(which, T, D, old, s, threadIdx.x);
    // The last word of a dim's older values holds the first new ones too: they are stored, by whichever wave,
    // once every such word has been written back.
    __syncthreads();
  }
  if (threadIdx.x == 0) *run.ep = (uint8_t)s;
  return KvqScale(s);
}

// a run by one wave
template <typename E>
__device__ __forceinline__ void kvq_append_run(const KvqAppendArgs& a, int which, const KvqRun<E>& run, int lane) {
  const int T = a.T, D = a.D;
  const int n = run.n, off = run.off, old = off > 0 ? *run.ep : 0;
  const bool vec = which ? a.vec_v : a.vec_k;  // 16-byte loads
  const float amax = vec ? kvq_amax<E, true>(run.src, run.ld, n, D, lane) : kvq_amax<E, false>(run.src, run.ld, n, D, lane);
  const int s = max(kvq_exponent(amax), old);
  run.template rescale<64>(which, T, D, old, s, lane);
  if (lane == 0) *run.ep = (uint8_t)s;
  const KvqScale sc(s);
  if (which) {
    if (vec) kvq_put_values<E, true>(run.src, run.ld, n, D, T, off, sc, run.blk, lane);
    else kvq_put_values<E, false>(run.src, run.ld, n, D, T, off, sc, run.blk, lane);
  } else {
    if (vec) kvq_put_keys<E, true>(run.src, run.ld, n, D, off, sc, run.blk, lane);
    else kvq_put_keys<E, false>(run.src, run.ld, n, D, off, sc, run.blk, lane);
  }
}

// A run by the workgroup's four waves, rows at 16-byte boundaries: a thread holds its elements
// between the maximum and the codes, so that the rows are read once.  red: five words.
template <typename E, int U>
__device__ __forceinline__ void kvq_keys_shared(const KvqRun<E>& run, int T, int D, uint32_t* red) {
  constexpr int N = 16 / (int)sizeof(E);
  typedef KvqVec<E, N, true> V;
  const int t = threadIdx.x, per = D / N, step = 256 / per, c = (t % per) * N, r0 = t / per;
  V x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = *(const V*)(run.src + kvq_row<true>(min(r0 + u * step, run.n - 1), run.ld) + c);
  float m = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, kvq_mag(kvq_ld(&x[u].v[e])));
  const KvqScale sc = kvq_shared_scale(run, 0, T, D, m, red);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + u * step;
    if (r < run.n) {
      KvqVec<uint32_t, N / 4, true> w;
#pragma unroll
      for (int e = 0; e < N / 4; ++e)
        w.v[e] = kvq_code4(kvq_fit(kvq_ld(&x[u].v[4 * e]), sc), kvq_fit(kvq_ld(&x[u].v[4 * e + 1]), sc),
                           kvq_fit(kvq_ld(&x[u].v[4 * e + 2]), sc), kvq_fit(kvq_ld(&x[u].v[4 * e + 3]), sc));
      *(KvqVec<uint32_t, N / 4, true>*)(run.blk + (size_t)(run.off + r) * D + c) = w;
    }
  }
}
template <typename E, int G>
__device__ __forceinline__ void kvq_values_shared(const KvqRun<E>& run, int T, int D, uint32_t* red) {
  typedef KvqVec<E, 2, true> V;
  const int t = threadIdx.x, per = D / 2, d = (t % per) * 2, off = run.off, end = off + run.n;
  const int first = (off & ~15) + 16 * (t / per), stride = 16 * (256 / per);
  V x[G][16];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int j = 0; j < 16; ++j)
      x[g][j] = *(const V*)(run.src + kvq_row<true>(min(max(first + g * stride + j - off, 0), run.n - 1), run.ld) + d);
  float m = 0.f;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int j = 0; j < 16; ++j) m = fmaxf(m, fmaxf(kvq_mag(kvq_ld(&x[g][j].v[0])), kvq_mag(kvq_ld(&x[g][j].v[1]))));
  const KvqScale sc = kvq_shared_scale(run, 1, T, D, m, red);
#pragma unroll
  for (int g = 0; g < G; ++g)
    if (first + g * stride < end)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float y[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = kvq_fit(kvq_ld(&x[g][j].v[e]), sc);
        kvq_put16(run.blk + (size_t)(d + e) * T, first + g * stride, off, end, y);
      }
}

// A workgroup takes one side (keys or values of a head) of a window of rows: the runs that start there.
// R: what a thread holds of a shared run covers 8192 R elements (a block has up to 128 x 128).
template <typename E, int R>
__global__ __launch_bounds__(256) void kvq_append_kernel(KvqAppendArgs a) {
  __shared__ uint32_t red[2][5];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // windows of rows fastest: the few that start a run in long prompts then fall on all XCDs alike
  const int windows = (a.n_rows + a.window - 1) / a.window, side = (int)(blockIdx.x / windows), which = side & 1, h = side >> 1;
  const int first = (int)(blockIdx.x % windows) * a.window;
  const int cap = a.n_blocks * a.T, last = a.n_rows - 1;
  // slots of the window's rows and of those that a run from it can reach (a block has at most 128),
  // read together; stop: the rows that do not continue the run before them
  int slot[3], prev[3];
  uint64_t stop[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int r = (int)min((long long)first + 64 * i + lane, (long long)last);
    slot[i] = a.slots[r], prev[i] = a.slots[max(r - 1, 0)];
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const long long r = (long long)first + 64 * i + lane;
    stop[i] = __ballot(r > last || r == 0 || (slot[i] & (a.T - 1)) == 0 || prev[i] != slot[i] - 1);
  }
  uint64_t m = stop[0] & __ballot(lane < a.window && (long long)first + lane <= last && slot[0] >= 0 && slot[0] < cap);
  const bool shared = (which ? a.vec_v : a.vec_k) && __builtin_popcountll(m) <= 2;
  for (int i = 0; m; m &= m - 1, ++i) {
    const int l = __builtin_ctzll(m), s0 = __builtin_amdgcn_readlane(slot[0], l);
    if (!shared && (i & 3) != wave) continue;
    // rows to the next one that starts anew
    const uint64_t rest = l < 63 ? stop[0] >> (l + 1) : 0;
    int n = 64 - l;
    if (rest) n = 1 + __builtin_ctzll(rest);
    else if (stop[1]) n += __builtin_ctzll(stop[1]);
    else n += 64 + (stop[2] ? __builtin_ctzll(stop[2]) : 64);
    const KvqRun<E> run(a, which, h, first + l, s0, n);
    if (!shared) kvq_append_run<E>(a, which, run, lane);
    else if (which) kvq_values_shared<E, R>(run, a.T, a.D, red[i & 1]);
    else kvq_keys_shared<E, R * (sizeof(E) == 2 ? 4 : 8)>(run, a.T, a.D, red[i & 1]);
  }
}

// Rows that a workgroup looks at: four while that makes few enough workgroups (each row may start a run, a
// step of single tokens), up to 64 for long prompts, where one in a block's rows does.  64 single
// tokens: 7.4 us a call with windows of 4, 16 with 16, 55 with 64; 16 prompts of up to 2048 rows: 116, 54, 41.
int kvq_append_window(int n_rows) { return std::max(4, std::min(64, n_rows / 1024 * 4)); }

void kvq_append(KvqAppendArgs a, hipStream_t st) {
  const int es = a.bf16 ? 2 : 4;
  // 16-byte loads, and 32 bits for an offset within a run (16 prompts of up to 2048 rows: 36 us, 59 by elements)
  a.vec_k = (((uintptr_t)a.k | a.ld_k * es) & 15) == 0 && a.ld_k < (1 << 22);
  a.vec_v = (((uintptr_t)a.v | a.ld_v * es) & 15) == 0 && a.ld_v < (1 << 22);
  a.window = kvq_append_window(a.n_rows);
  const dim3 grid((unsigned)((a.n_rows + a.window - 1) / a.window) * a.Hkv * 2);
  const bool two = a.T * a.D > 64 * 128;
  auto kernel = a.bf16 ? two ? kvq_append_kernel<uint16_t, 2> : kvq_append_kernel<uint16_t, 1>
                       : two ? kvq_append_kernel<float, 2> : kvq_append_kernel<float, 1>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
}

// ---------------- attention ----------------
// Request b has rows cu[b] .. cu[b + 1] - 1 of q, its newest positions: row i of
// n sits at position len - n + i and sees the keys at [0, that position].  A
// position whose table entry is no block of the cache is seen by none; a row
// that sees nothing gets zeros.
//
// The rows of a request that share a KV head (i * g + head in group, g = query heads
// a KV head) are the columns of 16-wide matrix products, S^T = K Q^T and O^T = V^T P^T,
// over steps of 64 keys, with a running maximum and sum.  Key 16 G + 4 t + i of a
// step is row 4 G + i of the t-th 16 x 16 tile of S^T, so lane group G (16 lanes)
// holds the weights of 16 consecutive keys of each query: these are the operand
// of the second product without a move, its V^T operand is 16 consecutive bytes of
// the value layout, and since blocks have at least 16 tokens all of them share
// one table entry and one scale.
//
// Keys are converted to bf16 with their scale (exact); bf16 queries are one
// operand, fp32 ones the sum of three (all 24 bits).  Weights are p = 2^(t - m) in fp32,
// t the score in the log2 domain.  fp32 calls split them into three bf16 operands like
// the queries, the values being bf16 with their scale.  bf16 calls have one operand:
// the weights take the value scale along, p' = 2^(t - m + e - R), e the value exponent of the
// key's block and R a running bound of t - m + e, so that the codes themselves, exact in fp16,
// are the other operand whatever the scales of different blocks are; p' is rounded to fp16,
// 11 bits where the output has 8 (8 x 64 rows are 0.00167 of their norm off the result in 64 bits, which rounded to bf16
// is 0.00166 off).  p' is formed alone, a lane's 16 of a step share e, so l takes
// their sum times 2^(R - e).  m and R follow their maxima lazily: only where a lane
// finds one grown by more than 2^8 are the maxima of all lanes taken and the sums rescaled.
//
// t - m + e - R is one multiply-add of a product and m - e + R while m is below 2^22.  Beyond, that sum and
// the rounding of t to fp32 are off by more than the exponent of a weight may be (equal scores of 3e7 gave infinite
// fp16 weights), so there t is rounded first, as m is, and the small terms join the difference.  Scores may be as large
// as fp32 holds.
typedef _Float16 kvq_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 kvq_h2 __attribute__((ext_vector_type(2)));

constexpr int KVQ_STEP = 64;
constexpr float KVQ_NONE = -3.4028234664e38f;  // m before the first key
constexpr float KVQ_FAR = 4194304.f;           // |m| from which differences are taken first
constexpr float KVQ_LAZY = 8.f;
constexpr float KVQ_LIFT = 6.f;     // p' of the largest lies at 2^6 (2^14 before R moves on): fp16 steps of 2^-30 of it

__device__ __forceinline__ bf16x8 kvq_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  bf16x8 r;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false),
               b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false),
               d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = c[0], r[5] = c[1], r[6] = d[0], r[7] = d[1];
  return r;
}
__device__ __forceinline__ kvq_h8 kvq_f16x8(uint32_t lo, uint32_t hi) {
  kvq_h8 r;
  const kvq_h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
  r[0] = a[0], r[1] = a[1], r[2] = b[0], r[3] = b[1], r[4] = c[0], r[5] = c[1], r[6] = d[0], r[7] = d[1];
  return r;
}

template <int D>
struct KvqStage {
  uint4 k[4][D / 64];  // 16 codes of key (tile t, row lane % 16), dims 64 u + 16 (lane / 16) ..
  uint4 v[D / 16];     // 16 keys of dim 16 dt + lane % 16
  int ek, ev;          // exponents of this lane's key rows and of its 16 keys
  bool has;            // its 16 keys begin inside the context, in a block of the cache
};

// Codes of positions that no row sees (key kend and on, blocks that are not there) may be
// anything: what is left of 16 codes from key `key` on, zero in their place.
struct KvqKeep {
  uint32_t m[4];
  __device__ __forceinline__ KvqKeep(int iev, int key, int kend) {
    const int n = iev < 0 ? 0 : kend - key;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int nb = n - 4 * w;
      m[w] = nb >= 4 ? ~0u : nb <= 0 ? 0u : (1u << (8 * nb)) - 1u;
    }
  }
  __device__ __forceinline__ uint4 operator()(uint4 v) const { return make_uint4(v.x & m[0], v.y & m[1], v.z & m[2], v.w & m[3]); }
};

// the operands of a step straight from a stage's codes; HALF: values as fp16 codes, else bf16 with their scale
template <int D, bool HALF>
struct KvqFromCodes {
  const KvqStage<D>& s;
  int ev, key, kend;
  __device__ __forceinline__ void keys(int t, int u, bf16x8& k0, bf16x8& k1) const {
    const float ks = kvq_pow2(s.ek - 127);
    k0 = kvq_bf16x8(s.k[t][u].x, s.k[t][u].y, ks);
    k1 = kvq_bf16x8(s.k[t][u].z, s.k[t][u].w, ks);
  }
  template <bool MASK, typename W8>
  __device__ __forceinline__ void values(int dt, W8& v0, W8& v1) const {
    uint4 v = s.v[dt];
    if constexpr (MASK) v = KvqKeep(ev, key, kend)(v);
    if constexpr (HALF) {
      v0 = kvq_f16x8(v.x, v.y);
      v1 = kvq_f16x8(v.z, v.w);
    } else {
      const float vs = kvq_pow2(max(ev, 1) - 127);
      v0 = kvq_bf16x8(v.x, v.y, vs);
      v1 = kvq_bf16x8(v.z, v.w, vs);
    }
  }
};

// where a lane's 16 keys of a step lie
struct KvqPlace {
  int k, v;  // table entries of the key rows' group and of the value group
};

template <int D>
struct KvqWalk {
  const KvqAttnArgs& a;
  const int* trow;
  int h, lane, kend, sh;  // sh: log2 of the block size
  size_t blk;             // bytes of one block of one side
  __device__ __forceinline__ KvqWalk(const KvqAttnArgs& args, int b, int head, int end)
      : a(args), trow(args.table + (size_t)b * args.width), h(head), lane(threadIdx.x & 63), kend(end),
        sh(__builtin_ctz(args.T)), blk((size_t)args.Hkv * args.T * D) {}
  // the table's entry for a position, and whether it is one (kept apart: a use of the loaded
  // value right behind the load would wait for it)
  __device__ __forceinline__ int entry(int key) const { return trow[min(key >> sh, a.width - 1)]; }
  __device__ __forceinline__ bool real(int p, int key) const { return key < kend && (unsigned)p < (unsigned)a.n_blocks; }
  __device__ __forceinline__ KvqPlace place(int j0) const {
    return KvqPlace{entry(j0 + 16 * ((lane & 15) >> 2)), entry(j0 + 16 * (lane >> 4))};
  }
  // a step's keys (with both exponents) and values; a missing block loads block 0 in its place, unused
  __device__ __forceinline__ void load_k(KvqStage<D>& s, int j0, const KvqPlace& pl) const {
    const int m = lane & 15, key = j0 + 16 * (m >> 2);
    const bool rk = real(pl.k, key);
    s.has = real(pl.v, j0 + 16 * (lane >> 4));
    const size_t pk = rk ? pl.k : 0, pv = s.has ? pl.v : 0;
    const uint8_t* kb = a.kc + pk * blk + (h * a.T + (key & (a.T - 1)) + (m & 3)) * D + 16 * (lane >> 4);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < D / 64; ++u) s.k[t][u] = *(const uint4*)(kb + 4 * t * D + 64 * u);
    s.ek = a.ke[pk * a.Hkv + h];
    s.ev = a.ve[pv * a.Hkv + h];
  }
  __device__ __forceinline__ void load_v(KvqStage<D>& s, int j0, const KvqPlace& pl) const {
    const int key = j0 + 16 * (lane >> 4);
    const size_t pv = real(pl.v, key) ? pl.v : 0;
    const uint8_t* vb = a.vc + pv * blk + (h * D + (lane & 15)) * a.T + (key & (a.T - 1));
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) s.v[dt] = *(const uint4*)(vb + 16 * dt * a.T);
  }
};

// a score in the log2 domain, rounded as one number, and what it lies above m: kept apart (fused, the
// product's rounding would be left over, more than an exponent holds where scores are large)
__device__ __forceinline__ float kvq_score(float s, float sc) {
#pragma clang fp contract(off)
  return s * sc;
}
__device__ __forceinline__ float kvq_above(float s, float sc, float m) {
#pragma clang fp contract(off)
  return s * sc - m;
}
// larger of two scores (the median with infinity: fmaxf would first quiet signalling NaNs, an instruction an operand)
__device__ __forceinline__ float kvq_max(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }
// largest over the four lane groups, in every lane
__device__ __forceinline__ float kvq_max_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// Running state of QT tiles of 16 query rows in one wave; PL operands carry a query and a weight (1: bf16 calls, 3: fp32).
template <int D, int QT, int PL>
struct KvqRows {
  static constexpr bool HALF = PL == 1;  // weights in fp16
  bf16x8 q[QT][PL][D / 32];
  floatx4 O[QT][D / 16];
  float m[QT], R[QT], l[QT];
  bool far[QT];    // |m| past KVQ_FAR in a lane (the same in the wave)
  int pos[QT];  // last position that this lane's row sees (-1: none)

  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      m[i] = KVQ_NONE;
      R[i] = l[i] = 0.f;
      far[i] = false;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) O[i][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // query operands of the tiles from rows of q (live: the row is one; else zeros): lane group c,
  // operand 2 u + w, element e is dim 64 u + 16 c + 8 w + e.  All loads go out first, and stand on no
  // branch of a lane: they would be waited for one by one.
  template <typename E>
  __device__ __forceinline__ void load_q(const E* const (&row)[QT], const bool (&live)[QT], bool neg, bool vec) {
    const int c = (threadIdx.x & 63) >> 4;
    E raw[QT][D / 32][8];
    if (vec) {
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int kd = 0; kd < D / 32; ++kd)
#pragma unroll
          for (int j = 0; j < 8; j += 16 / (int)sizeof(E))
            *(uint4*)(raw[i][kd] + j) = *(const uint4*)(row[i] + 64 * (kd >> 1) + 16 * c + 8 * (kd & 1) + j);
    } else {
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int kd = 0; kd < D / 32; ++kd)
#pragma unroll
          for (int e = 0; e < 8; ++e) raw[i][kd][e] = row[i][64 * (kd >> 1) + 16 * c + 8 * (kd & 1) + e];
    }
#pragma unroll
    for (int i = 0; i < QT; ++i)
#pragma unroll
      for (int kd = 0; kd < D / 32; ++kd) {
        if constexpr (HALF) {
          const uint32_t flip = neg ? 0x80008000u : 0u;
          uint4 x = __builtin_bit_cast(uint4, raw[i][kd]);
          x = live[i] ? make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip) : make_uint4(0, 0, 0, 0);
          q[i][0][kd] = __builtin_bit_cast(bf16x8, x);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x = live[i] ? raw[i][kd][e] : 0.f;
            if (neg) x = -x;
#pragma unroll
            for (int pl = 0; pl < PL; ++pl) {  // (the last rounding of three takes what is left: 24 bits)
              uint16_t b = f2bf(x);
              if (pl == 0 && (b & 0x7FFF) == 0x7F80 && fabsf(x) < INFINITY) --b;  // rounded past the largest bf16: that one
              q[i][pl][kd][e] = __builtin_bit_cast(__bf16, b);
              x -= bf2f(b);
            }
          }
        }
      }
  }

  // what takes the sums from R (and the codes' exponents) to m
  __device__ __forceinline__ float to_m(int i) const { return HALF ? exp2f(R[i] - 127.f) : 1.f; }

  // one step: keys j0 .. j0 + 63, their operands from src, iev the value exponent of this lane's keys
  // (scored(): the key operands are free)
  struct Nothing {
    __device__ __forceinline__ void operator()() const {}
  };
  template <bool MASK, typename Src, typename Scored = Nothing>
  __device__ __forceinline__ void step(const Src& src, int iev, int j0, int kend, float sc, Scored scored = Scored{}) {
    const int c = (threadIdx.x & 63) >> 4;
    floatx4 S[QT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      bf16x8 k[D / 32];
#pragma unroll
      for (int u = 0; u < D / 64; ++u) src.keys(t, u, k[2 * u], k[2 * u + 1]);
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        S[i][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int pl = PL - 1; pl >= 0; --pl)  // small parts first
#pragma unroll
          for (int kd = 0; kd < D / 32; ++kd)
            S[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[kd], q[i][pl][kd], S[i][t], 0, 0, 0);
      }
    }
    scored();
    typedef std::conditional_t<HALF, kvq_h8, bf16x8> W8;
    W8 P[QT][PL][2];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      if constexpr (MASK) {
        const int last = (iev < 0 ? -1 : min(pos[i], kend - 1)) - (j0 + 16 * c);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[i][t][e] = 4 * t + e <= last ? S[i][t][e] : -INFINITY;
      }
      float x = S[i][0][0];
#pragma unroll
      for (int j = 1; j < 16; ++j) x = kvq_max(x, S[i][j >> 2][j & 3]);
      x = kvq_score(x, sc);
      // e - R (0 for a block that is not there, whose scores are -inf)
      float ev = 0.f;
      if (HALF && (!MASK || iev >= 0)) ev = (float)iev - R[i];
      if (__builtin_expect(far[i] | (__ballot(x > m[i] + (HALF ? fminf(KVQ_LAZY, KVQ_LAZY + KVQ_LIFT - ev) : KVQ_LAZY)) != 0), 0)) {
        const float mn = fmaxf(m[i], kvq_max_groups(x)), down = m[i] - mn;
        float fr = down;
        if constexpr (HALF) {
          const float up = fmaxf(down, kvq_max_groups(x - mn + ev) - KVQ_LIFT);  // R's move
          R[i] += up;
          if (!MASK || iev >= 0) ev -= up;
          fr -= up;
        }
        fr = exp2f(fr);
        l[i] *= exp2f(down);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) O[i][dt] *= fr;
        m[i] = mn;
        far[i] = __any(fabsf(mn) > KVQ_FAR && mn > KVQ_NONE);
        if (far[i]) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[i][t][e] = kvq_above(S[i][t][e], sc, mn);
        }
      }
      // exponents of p: S f + at; of p': S f + off
      const float f = far[i] ? 1.f : sc, at = far[i] ? 0.f : -m[i], off = ev + at;
      float ls = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(S[i][t][e], f, off));
          ls += p[e];
        }
#pragma unroll
        for (int pl = 0; pl < PL; ++pl)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const auto w = __builtin_convertvector(kvq_f2{p[e], p[e + 1]}, std::conditional_t<HALF, kvq_h2, bf16x2>);
            P[i][pl][t >> 1][4 * (t & 1) + e] = w[0];
            P[i][pl][t >> 1][4 * (t & 1) + e + 1] = w[1];
            if (pl + 1 < PL) {
              p[e] -= (float)w[0];
              p[e + 1] -= (float)w[1];
            }
          }
      }
      if constexpr (HALF) {
        ls *= __builtin_amdgcn_exp2f(-ev);  // from p' to p
        // values 2^60 below what the largest p' stands for (blocks of zeros): p' may have
        // left fp32's range where p has not
        if (__any(ev < -60.f)) {
          float ps = 0.f;
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) ps += __builtin_amdgcn_exp2f(fmaf(S[i][t][e], f, at));
          ls = ps;
        }
      }
      l[i] += ls;
    }
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      W8 v0, v1;
      src.template values<MASK>(dt, v0, v1);
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int pl = PL - 1; pl >= 0; --pl) {
          if constexpr (HALF) {
            O[i][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, P[i][pl][0], O[i][dt], 0, 0, 0);
            O[i][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, P[i][pl][1], O[i][dt], 0, 0, 0);
          } else {
            O[i][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, P[i][pl][0], O[i][dt], 0, 0, 0);
            O[i][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, P[i][pl][1], O[i][dt], 0, 0, 0);
          }
        }
    }
  }
};

// Rows and keys of one request under a launch: the same arithmetic in the attention and the merge kernel.
struct KvqGeom {
  int r0, n;       // first row of q, rows (at most max_q)
  int n_rows;
  int first;       // position of row 0
  int chunk;       // keys of a split
  int limit;       // positions that exist for the table
  __device__ __forceinline__ KvqGeom(const KvqAttnArgs& a, int b) {
    const int c0 = a.cu[b], len = a.lens[b];
    const long long all = (long long)a.cu[b + 1] - c0, f = (long long)len - all;
    r0 = c0;
    n_rows = a.n_rows;
    n = (int)max(0ll, min(all, (long long)a.max_q));
    first = (int)max(f, (long long)INT_MIN / 2);
    limit = (int)max(0ll, min((long long)a.width * a.T, (long long)len));
    chunk = max(a.chunk, ((limit + a.nsplit - 1) / a.nsplit + KVQ_STEP - 1) & ~(KVQ_STEP - 1));
  }
  // row i is one of q's
  __device__ __forceinline__ bool has(int i) const { return (unsigned long long)((long long)r0 + i) < (unsigned long long)n_rows; }
  // keys seen by the last row of rows [r, r + rows) of the request's n * g
  __device__ __forceinline__ int keys(int r, int rows, int g) const {
    const int last = min(r + rows, n * g) - 1;
    return max(0, min(limit, first + last / g + 1));
  }
};

// Waves split the keys: a workgroup of four owns 16 QT rows of one (request, KV head)
// and one share of its keys; wave w takes every fourth step, a step's codes in
// registers while the next step's are on their way, and the four meet in LDS.
// For few rows, where the cache's bytes bound it: single tokens of 64 requests of up to 16384, 8 heads
// of 128, 1296 MB in 243 us, 5.3 TB/s (a large copy reads and writes 5.1 to 5.2); a single request of 412
// is latency (7.7 us a call).
template <typename E, int D, int QT>
__global__ __launch_bounds__(256) void kvq_attn_keys_kernel(KvqAttnArgs a) {
  constexpr int ROWS = 16 * QT, RS = D + 4;
  __shared__ __align__(16) float so[4 * ROWS * RS];
  __shared__ float sm[4 * ROWS], sl[4 * ROWS];
  const int g = a.Hq / a.Hkv;
  int w = blockIdx.x;
  const int h = w % a.Hkv;
  w /= a.Hkv;
  const int grp = w % a.groups;
  w /= a.groups;
  const int split = w % a.nsplit, b = w / a.nsplit;
  const KvqGeom ge(a, b);
  const int R = ge.n * g, rb = grp * ROWS;
  if (rb >= R) return;
  const int kall = ge.keys(rb, ROWS, g), active = max(1, (kall + ge.chunk - 1) / ge.chunk);
  if (split >= active) return;
  const int kbeg = split * ge.chunk, kend = min(kbeg + ge.chunk, kall);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 15, c = lane >> 4;
  const float sc = a.scale_log2;
  KvqRows<D, QT, sizeof(E) == 2 ? 1 : 3> rows;
  rows.start();
  {
    const E* row[QT];
    bool live[QT];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int r = rb + 16 * i + col, n = r / g;
      live[i] = r < R && ge.has(n);
      rows.pos[i] = live[i] ? ge.first + n : -1;
      row[i] = (const E*)a.q + (live[i] ? (size_t)(ge.r0 + n) : 0) * a.ld_q + (size_t)(h * g + (r - n * g)) * D;
    }
    rows.load_q(row, live, a.neg, a.vec);
  }
  const int seen_all = min(kend, ge.first + rb / g + 1);  // keys below this are seen by every row
  const KvqWalk<D> walk(a, b, h, kend);
  const int first = kbeg + wave * KVQ_STEP, nit = first < kend ? (kend - first + 4 * KVQ_STEP - 1) / (4 * KVQ_STEP) : 0;
  auto key = [&](int it) { return first + it * 4 * KVQ_STEP; };
  if (nit > 0) {
    KvqStage<D> s;
    KvqPlace pl = walk.place(key(0)), next = walk.place(key(1));
    walk.load_k(s, key(0), pl);
    walk.load_v(s, key(0), pl);
    int it = 0;
    // one stage of registers: the next step's keys are asked for once this step's scores are
    // there, its values once they are summed
    auto step = [&](auto mask) {
      const int ev = s.has ? s.ev : -1;
      pl = next;
      next = walk.place(key(it + 2));
      rows.template step<decltype(mask)::value>(KvqFromCodes<D, sizeof(E) == 2>{s, ev, key(it) + 16 * c, kend}, ev, key(it), kend,
                                                sc, [&] { walk.load_k(s, key(it + 1), pl); });
      walk.load_v(s, key(it + 1), pl);
      ++it;
    };
    // steps that every row sees whole come first, without a mask (two loops, not a branch a step,
    // keep the accumulators in place)
    const int whole = min(nit, (seen_all - first + 3 * KVQ_STEP) / (4 * KVQ_STEP));
    while (it < whole && __all(s.has)) step(std::false_type{});
    while (it < nit) step(std::true_type{});
  }
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float l = rows.l[i];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const float f = rows.to_m(i);
    float* row = so + (size_t)(wave * ROWS + 16 * i + col) * RS;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *(floatx4*)(row + 16 * dt + 4 * c) = rows.O[i][dt] * f;
    if (c == 0) {
      sm[wave * ROWS + 16 * i + col] = rows.m[i];
      sl[wave * ROWS + 16 * i + col] = l;
    }
  }
  __syncthreads();
  const size_t part = (((size_t)b * a.Hkv + h) * a.nsplit + split) * a.rows_pad + rb;
  for (int i = tid; i < ROWS * (D / 4); i += 256) {
    const int r = i / (D / 4), d = 4 * (i % (D / 4));
    if (rb + r >= R || !ge.has((rb + r) / g)) continue;
    float M = sm[r];
#pragma unroll
    for (int v = 1; v < 4; ++v) M = fmaxf(M, sm[v * ROWS + r]);
    float L = 0.f;
    floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float e = exp2f(sm[v * ROWS + r] - M);
      L += sl[v * ROWS + r] * e;
      o += *(const floatx4*)(so + (size_t)(v * ROWS + r) * RS + d) * e;
    }
    if (active == 1) {
      kvq_store4((E*)a.o + (size_t)(ge.r0 + (rb + r) / g) * a.ld_o + (size_t)(h * g + (rb + r) % g) * D + d, o, L);
    } else {
      *(floatx4*)(a.part_o + (part + r) * D + d) = o;
      if (d == 0) a.part_s[part + r] = make_float2(M, L);
    }
  }
}

// Waves split the rows: a workgroup of NW waves owns 32 NW rows of one (request, KV head)
// and one share of its keys.  A step's codes are converted once for all waves, half
// of them the keys and half the values, into operands in LDS (32 KB at D = 128, two
// steps' worth), while the codes of the next two steps are on their way in
// registers; every wave multiplies the whole step with its own two tiles of 16
// rows.  bf16 calls with many rows.  8 x 64 rows of 32 heads, contexts to 4352 (19.6 GFLOP): 47 us
// a call; under a trace, which adds some, 43 this kernel and 8 the merge.  A step takes a workgroup 1.4 to 1.7 us, of which
// the products are 0.85 at the matrix cores' peak, and the longest context's shares have 14: 20 to 24 us.  The
// rest of the kernel is the first codes' way in, the parts of the shares (28 MB out, 5 us at the rate of a large copy) and the
// workgroups that start late.  Running the next
// step's first product under the exponentials (interleaved one to four instructions) measured the same.
template <int D>
struct KvqFromLds {
  const uint16_t* st;  // operands of 64 x 16 bytes: keys (t, kd), then values (dt, half)
  int lane;
  __device__ __forceinline__ void keys(int t, int u, bf16x8& k0, bf16x8& k1) const {
    const uint16_t* p = st + ((t * (D / 32) + 2 * u) * 64 + lane) * 8;
    k0 = *(const bf16x8*)p;
    k1 = *(const bf16x8*)(p + 512);
  }
  template <bool MASK>
  __device__ __forceinline__ void values(int dt, kvq_h8& v0, kvq_h8& v1) const {
    const uint16_t* p = st + ((4 * (D / 32) + 2 * dt) * 64 + lane) * 8;
    v0 = *(const kvq_h8*)p;
    v1 = *(const kvq_h8*)(p + 512);
  }
};

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kvq_attn_rows_kernel(KvqAttnArgs a) {
  constexpr int QT = 2, WROWS = 16 * QT, ROWS = NW * WROWS;
  constexpr int PIECES = D / 16;            // 1 KiB of codes each, of a step's keys and of its values
  constexpr int MINE = 2 * PIECES / NW;     // of this wave: keys (waves below NW / 2) or values
  constexpr int STAGE = 4 * PIECES * 512;   // elements of a step's operands
  __shared__ __align__(16) uint16_t sm[2 * STAGE];
  const int g = a.Hq / a.Hkv;
  int w = blockIdx.x;
  const int h = w % a.Hkv;
  w /= a.Hkv;
  const int grp = w % a.groups;
  w /= a.groups;
  const int split = w % a.nsplit, b = w / a.nsplit;
  const KvqGeom ge(a, b);
  const int R = ge.n * g, rb = grp * ROWS;
  if (rb >= R) return;
  const int kall = ge.keys(rb, ROWS, g), active = max(1, (kall + ge.chunk - 1) / ge.chunk);
  if (split >= active) return;
  const int kbeg = split * ge.chunk, kend = min(kbeg + ge.chunk, kall);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, c = lane >> 4;
  const float sc = a.scale_log2;
  const KvqWalk<D> walk(a, b, h, kend);
  const int nit = (kend - kbeg + KVQ_STEP - 1) / KVQ_STEP;
  // this wave's share of a step: pieces at base + i * stride
  const bool of_v = wave >= NW / 2;
  const int first_piece = (of_v ? wave - NW / 2 : wave) * MINE;
  const int group = of_v ? c : col >> 2;  // of the 16 keys in which its lanes' codes lie
  const uint8_t* const side = of_v ? a.vc : a.kc;
  constexpr int U = D / 64;  // pieces of a key tile
  static_assert(MINE == 1 || MINE % U == 0, "a wave's pieces start at a tile's first or are one");
  struct Raw {
    uint4 x[MINE];
    int ek, ev;
    bool has;
    __device__ __forceinline__ int exp_v() const { return has ? ev : -1; }
  };
  struct Two {
    int data, v;  // table entries of the codes' and of this lane's 16 keys
  };
  auto place = [&](int j0) { return Two{walk.entry(j0 + 16 * group), walk.entry(j0 + 16 * c)}; };
  // pl: the entries of these keys, and then those of two steps further on (asked for before the codes:
  // loads come back in order)
  auto load = [&](Raw& r, int j0, Two& pl) {
    // (one address and no branch for both roles: loads on a branch are waited for at its end)
    const int at = (j0 + 16 * group) & (a.T - 1);
    const int off = of_v ? (h * D + 16 * first_piece + col) * a.T + at
                         : (h * a.T + at + (col & 3) + 4 * (first_piece / U)) * D + 64 * (first_piece % U) + 16 * c;
    r.has = walk.real(pl.v, j0 + 16 * c);
    const size_t blk = walk.real(pl.data, j0 + 16 * group) ? pl.data : 0, bv = r.has ? pl.v : 0;
    pl = place(j0 + 2 * KVQ_STEP);
    const uint8_t* p = side + blk * walk.blk + off;
#pragma unroll
    for (int i = 0; i < MINE; ++i) r.x[i] = *(const uint4*)(p + (of_v ? 16 * i * a.T : 4 * (i / U) * D + 64 * (i % U)));
    r.ek = a.ke[blk * a.Hkv + h];
    r.ev = a.ve[bv * a.Hkv + h];
  };
  auto store = [&](const Raw& r, int j0, uint16_t* st) {
    uint16_t* p = st + ((of_v ? 2 * PIECES : 0) + 2 * first_piece) * 512 + lane * 8;
    if (of_v) {
      const KvqKeep keep(r.exp_v(), j0 + 16 * c, kend);
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const uint4 v = keep(r.x[i]);
        *(kvq_h8*)(p + 1024 * i) = kvq_f16x8(v.x, v.y);
        *(kvq_h8*)(p + 1024 * i + 512) = kvq_f16x8(v.z, v.w);
      }
    } else {
      const float ks = kvq_pow2(r.ek - 127);
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        *(bf16x8*)(p + 1024 * i) = kvq_bf16x8(r.x[i].x, r.x[i].y, ks);
        *(bf16x8*)(p + 1024 * i + 512) = kvq_bf16x8(r.x[i].z, r.x[i].w, ks);
      }
    }
  };
  auto key = [&](int it) { return kbeg + it * KVQ_STEP; };
  Raw ra, rb2;
  Two pa = place(key(0)), pb = place(key(1));
  load(ra, key(0), pa);
  // (of two waves on a SIMD the one goes first: they take turns at the matrix core and the exponentials,
  // 49.7 us in place of 52.6 for 8 x 64 rows at contexts to 4352; one wave a SIMD has no other)
  if (NW == 8 && wave < NW / 2) __builtin_amdgcn_s_setprio(1);
  KvqRows<D, QT, 1> rows;
  rows.start();
  const int wr = rb + wave * WROWS;
  {
    const uint16_t* row[QT];
    bool live[QT];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int r = wr + 16 * i + col, n = r / g;
      live[i] = r < R && ge.has(n);
      rows.pos[i] = live[i] ? ge.first + n : -1;
      row[i] = (const uint16_t*)a.q + (live[i] ? (size_t)(ge.r0 + n) : 0) * a.ld_q + (size_t)(h * g + (r - n * g)) * D;
    }
    rows.load_q(row, live, a.neg, a.vec);
  }
  const int seen_all = min(kend, ge.first + min(wr, R - 1) / g + 1);  // keys below this are seen by every row of the wave
  if (nit > 0) {
    load(rb2, key(1), pb);
    store(ra, key(0), sm);
    int ev_now = ra.exp_v(), it = 0;
    load(ra, key(2), pa);
    // step `it` from stage it & 1; r holds the codes of step it + 1, and takes those of it + 3
    auto step = [&](auto mask, auto odd, Raw& r, Two& pl) {
      constexpr int O = decltype(odd)::value;
      lds_barrier();  // step it is in its stage, and every wave is done with the other
      const int ev_next = r.exp_v();
      store(r, key(it + 1), sm + (O ? 0 : STAGE));
      load(r, key(it + 3), pl);
      rows.template step<decltype(mask)::value>(KvqFromLds<D>{sm + (O ? STAGE : 0), lane}, ev_now, key(it), kend, sc);
      ev_now = ev_next;
      ++it;
    };
    // pairs of steps that every row of the wave sees whole come first, without a mask (two
    // loops, not a branch a step, keep the accumulators in place)
    const int whole = min(nit, (seen_all - kbeg) / KVQ_STEP) - 1;
    while (it < whole && __all(ev_now >= 0 && rb2.has)) {
      step(std::false_type{}, std::integral_constant<int, 0>{}, rb2, pb);
      step(std::false_type{}, std::integral_constant<int, 1>{}, ra, pa);
    }
    while (it < nit) {
      step(std::true_type{}, std::integral_constant<int, 0>{}, rb2, pb);
      if (it < nit) step(std::true_type{}, std::integral_constant<int, 1>{}, ra, pa);
    }
  }
  const size_t part = (((size_t)b * a.Hkv + h) * a.nsplit + split) * a.rows_pad;
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    float l = rows.l[i];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const float f = rows.to_m(i);
    const int r = wr + 16 * i + col;
    if (r >= R || !ge.has(r / g)) continue;
    if (active == 1) {
      uint16_t* dst = (uint16_t*)a.o + (size_t)(ge.r0 + r / g) * a.ld_o + (size_t)(h * g + r % g) * D + 4 * c;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) kvq_store4(dst + 16 * dt, rows.O[i][dt] * f, l);
    } else {
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) *(floatx4*)(a.part_o + (part + r) * D + 16 * dt + 4 * c) = rows.O[i][dt] * f;
      if (c == 0) a.part_s[part + r] = make_float2(rows.m[i], l);
    }
  }
}

// Joins the splits of rows that have more than one: D / 4 lanes a row and query head,
// four splits' loads in flight together.  Bound by the bytes of the partial sums (28 MB in 8 us).
template <typename E, int D>
__global__ __launch_bounds__(256) void kvq_merge_kernel(KvqAttnArgs a) {
  constexpr int LANES = D / 4;
  const int g = a.Hq / a.Hkv, rows = a.max_q * g, d = 4 * (threadIdx.x % LANES);
  const unsigned w = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const int r = (int)(w % rows), h = (int)(w / rows % a.Hkv), b = (int)(w / rows / a.Hkv);
  if (b >= a.B) return;
  const KvqGeom ge(a, b);
  if (r >= ge.n * g || !ge.has(r / g)) return;
  const int kall = ge.keys(r / a.group_rows * a.group_rows, a.group_rows, g), active = (kall + ge.chunk - 1) / ge.chunk;
  if (active <= 1) return;
  const size_t part = ((size_t)b * a.Hkv + h) * a.nsplit * a.rows_pad + r;
  float M = KVQ_NONE, L = 0.f;
  floatx4 o = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < active; s += 4) {
    float2 st[4];
    floatx4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // (past the last: that one again, without weight)
      const size_t at = part + (size_t)min(s + j, active - 1) * a.rows_pad;
      st[j] = a.part_s[at];
      v[j] = *(const floatx4*)(a.part_o + at * D + d);
    }
    const float m = fmaxf(M, fmaxf(fmaxf(st[0].x, st[1].x), fmaxf(st[2].x, st[3].x)));
    const float f = exp2f(M - m);
    L *= f;
    o *= f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float e = s + j < active ? exp2f(st[j].x - m) : 0.f;
      L = fmaf(st[j].y, e, L);
      o += v[j] * e;
    }
    M = m;
  }
  kvq_store4((E*)a.o + (size_t)(ge.r0 + r / g) * a.ld_o + (size_t)(h * g + r % g) * D + d, o, L);
}

// How a call is split (host): the kernel, rows of a workgroup and shares of the keys with the least
// cost by a model of the longest context.
//
// Waves that split the keys (16 or 32 rows a workgroup; all fp32 calls): a round is 256 keys, 1.4 us
// (1.0 at D = 64, 1.65 for 32 rows at D = 128) while the workgroups draw less than the HBM gives; rounds
// in turn beyond about 200 workgroups (256: what the card holds of the widest), for contexts
// are ragged and not all have their longest.  Waves that split the rows (256 or 128 a workgroup): a
// round is 64 keys, 1.75 us up to 340 workgroups of eight waves or 680 of four, and 2 us for the start.  A second share
// adds the merge: its launch, and a part for each share.
//
// 340 and 680 are more than the card holds at D = 128 (256 and 512 at 220 and 236 registers): with ragged contexts some
// shares are empty.  Requests of one length pay for that, since the workgroups past 256 then run after the others:
// 8 of 4352, 64 tokens: 82 us (36 GFLOP; ragged 47, 20 GFLOP), 16 of 2064: 74 (34 GFLOP; ragged 66, 19 GFLOP).  D = 64 takes
// the step of D = 128: it was not fitted (8 of 4352, 64 tokens: 36 us ragged, 59 of one length).  The causal triangle
// of a prompt counts as its longest row too: 2048 tokens 70 us.
//
// Measured (us a call, 8B heads, contexts ragged up to the length; keys split, 128 and 256 rows
// a workgroup): 8 requests of 1000, 64 tokens: 26, 33, 33; 8 of 4000, 33 tokens: 33, 43, 40; 8 of
// 4288, 64 tokens: 54, 49, 46; 8 of 4000, 80 tokens: 54, 52, 58; 32 of 2000, 64 tokens: 119,
// 75, 73; a prompt of 2048: 114, 69, 72.  Shares: one token at 16000 keys 15.0 with 32, 87 with
// one; 64 tokens at up to 8000: 126 with one, 132 to 189 with 2 to 32.
void kvq_attn_plan(KvqAttnArgs& a) {
  const int rows = a.max_q * (a.Hq / a.Hkv);
  a.qt = rows > 16 && a.bf16 ? 2 : 1;
  double best = 0.0;
  int round = 0;
  for (int by_rows : {0, 8, 4}) {
    if (by_rows && !a.bf16) break;
    const int group_rows = by_rows ? 32 * by_rows : 16 * a.qt, groups = (rows + group_rows - 1) / group_rows;
    const double base = (double)a.B * a.Hkv * groups;
    const int keys = by_rows ? KVQ_STEP : 4 * KVQ_STEP;
    const long long rounds = (a.max_len + keys - 1) / keys;
    const bool wide = a.qt == 2 && a.D == 128;
    const double one = by_rows ? 1.75 : a.D == 64 ? 1.0 : wide ? 1.65 : 1.4;
    const double fit = by_rows ? 2720.0 / by_rows : wide ? 256.0 : 200.0;
    for (int n = 1; n <= 64 && n <= rounds; ++n) {
      const double us = (rounds + n - 1) / n * one * std::max(1.0, base * n / fit) +
                        (n > 1 ? 2.5 + 0.25 * n + base * n * group_rows * a.D * 1e-6 : 0.0) + (by_rows ? 2.0 : 0.0);
      if (round == 0 || us < best) {
        best = us;
        round = keys;
        a.by_rows = by_rows;
        a.group_rows = group_rows;
        a.groups = groups;
        a.nsplit = n;
      }
    }
  }
  const long long rounds = (a.max_len + round - 1) / round;
  a.rows_pad = a.groups * a.group_rows;
  a.chunk = (int)((rounds + a.nsplit - 1) / a.nsplit) * round;
  a.nsplit = (a.max_len + a.chunk - 1) / a.chunk;
}

static size_t kvq_part_rows(const KvqAttnArgs& a) { return (size_t)a.B * a.Hkv * a.nsplit * a.rows_pad; }

size_t kvq_attn_workspace(KvqAttnArgs a) {
  kvq_attn_plan(a);
  return a.nsplit > 1 ? kvq_part_rows(a) * (a.D + 2) * 4 : 0;
}

template <typename E, int D>
static void kvq_launch(const KvqAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.B * a.nsplit * a.groups * a.Hkv));
  if constexpr (sizeof(E) == 2) {
    if (a.by_rows == 8) hipLaunchKernelGGL((kvq_attn_rows_kernel<D, 8>), grid, dim3(512), 0, st, a);
    else if (a.by_rows) hipLaunchKernelGGL((kvq_attn_rows_kernel<D, 4>), grid, dim3(256), 0, st, a);
    else if (a.qt == 2) hipLaunchKernelGGL((kvq_attn_keys_kernel<E, D, 2>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kvq_attn_keys_kernel<E, D, 1>), grid, dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL((kvq_attn_keys_kernel<E, D, 1>), grid, dim3(256), 0, st, a);
  }
  if (a.nsplit > 1) {
    const long long rows = (long long)a.B * a.Hkv * a.max_q * (a.Hq / a.Hkv);
    hipLaunchKernelGGL((kvq_merge_kernel<E, D>), dim3((unsigned)((rows * (D / 4) + 255) / 256)), dim3(256), 0, st, a);
  }
}

void kvq_attention(KvqAttnArgs a, hipStream_t st) {
  kvq_attn_plan(a);
  a.part_o = (float*)a.workspace;
  a.part_s = (float2*)(a.part_o + kvq_part_rows(a) * a.D);
  // a negative scale turns the queries' signs
  a.neg = a.scale < 0.0;
  // rows start on 16 bytes, heads then do (8 x 64 rows of 32 heads: 47 us, 51 by elements)
  a.vec = (((uintptr_t)a.q | a.ld_q * (a.bf16 ? 2 : 4)) & 15) == 0;
  // a zero scale: the smallest number in its place, whose scores are below 2^-21 (0 * -inf is none where a key is hidden)
  a.scale_log2 = std::max(kvq_scale_log2(a.scale), 0x1p-149f);
  if (a.bf16) {
    if (a.D == 128) kvq_launch<uint16_t, 128>(a, st);
    else kvq_launch<uint16_t, 64>(a, st);
  } else {
    if (a.D == 128) kvq_launch<float, 128>(a, st);
    else kvq_launch<float, 64>(a, st);
  }
}

}  // namespace ssd
