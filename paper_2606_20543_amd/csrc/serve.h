// Serving operators that stand beside the verify pass: block tables and slot
// maps from request lengths, and rotary positions with several axes
// (device code and launchers, included by kernels_misc.hip).
#pragma once

#include "ssd_internal.h"

namespace ssd {

// ---------------- block tables and slot maps ----------------
// Request b holds held_b tokens and gets fresh_b more.  With T tokens a block it has
// ceil(held / T) blocks and needs ceil((held + fresh) / T); the blocks that the
// requests lack come from the pool in request order, so the first of request b
// is pool[sum of the lacks before b].  A workgroup owns SLOT_SEQS requests and
// sums the lengths of all requests before them itself (a few loads a thread),
// so one launch does it with no hand-off between workgroups; several share the rows
// of the same requests where there are many.  (More than some thousand requests take four launches.)  Bound by its
// launch and three dependent round trips (lengths, table or pool entry, store): 64
// requests of one new token 7.6 us a call (5.3 the kernel), 2048 of up to 64 7.7.
constexpr int SLOT_T = 256, SLOT_SEQS = 8;
constexpr int SLOT_ALONE = 8192;  // most requests of the single launch

__device__ __forceinline__ long long wave_sum_ll(long long v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// blocks of n tokens, at most the table's width
__device__ __forceinline__ int slot_blocks(long long n, int T, int sh, int width) {
  const long long c = (n + T - 1) >> sh;
  return (int)(c < width ? c : width);
}

__global__ __launch_bounds__(SLOT_T) void slots_kernel(SlotArgs a) {
  __shared__ long long red[3][SLOT_T / 64];
  __shared__ int s_held[SLOT_SEQS], s_have[SLOT_SEQS];
  __shared__ long long s_start[SLOT_SEQS + 1], s_cu[SLOT_SEQS + 1], s_all;
  const int tid = threadIdx.x, b0 = blockIdx.x * SLOT_SEQS, nb = min(SLOT_SEQS, a.B - b0);
  const int T = a.T, W = a.width, sh = __builtin_ctz(a.T);  // (T is a power of two)
  const bool head = blockIdx.y == 0;  // writes what is not a row's
  // rows and lacking blocks of the requests before this workgroup's, rows of all
  long long rows = 0, lack = 0, all = 0;
  for (int b = tid; b < a.B; b += SLOT_T) {
    const long long h = max(a.held[b], 0), n = max(a.fresh[b], 0);
    all += n;
    if (b < b0) {
      rows += n;
      lack += slot_blocks(h + n, T, sh, W) - slot_blocks(h, T, sh, W);
    }
  }
  rows = wave_sum_ll(rows);
  lack = wave_sum_ll(lack);
  all = wave_sum_ll(all);
  if ((tid & 63) == 0) {
    red[0][tid >> 6] = rows;
    red[1][tid >> 6] = lack;
    red[2][tid >> 6] = all;
  }
  __syncthreads();
  if (tid == 0) {
    long long r = 0, l = 0, t = 0;
    for (int w = 0; w < SLOT_T / 64; ++w) {
      r += red[0][w];
      l += red[1][w];
      t += red[2][w];
    }
    s_all = t;
    if (head && b0 == 0) a.cu[0] = 0;
    for (int i = 0; i < nb; ++i) {
      const long long h = max(a.held[b0 + i], 0), n = max(a.fresh[b0 + i], 0);
      s_held[i] = (int)h;
      s_have[i] = slot_blocks(h, T, sh, W);
      s_cu[i] = r;
      s_start[i] = l;
      r += n;
      l += slot_blocks(h + n, T, sh, W) - s_have[i];
      if (head) {
        a.cu[b0 + i + 1] = (int)(r < INT_MAX ? r : INT_MAX);
        a.lens[b0 + i] = (int)(h + n < INT_MAX ? h + n : INT_MAX);
      }
    }
    s_cu[nb] = r;
    s_start[nb] = l;
    if (head && b0 + nb == a.B) a.used[0] = (int)(l < INT_MAX ? l : INT_MAX);
  }
  __syncthreads();
  // table entries of the blocks taken here (an empty pool leaves -1)
  auto pooled = [&](long long i) { return i < a.n_pool ? a.pool[i] : -1; };
  for (long long e = s_start[0] + tid; head && e < s_start[nb]; e += SLOT_T) {
    int i = 0;
    while (s_start[i + 1] <= e) ++i;
    a.table[(size_t)(b0 + i) * W + s_have[i] + (e - s_start[i])] = pooled(e);
  }
  // new rows
  const long long last = min(s_cu[nb], (long long)a.n_rows);
  for (long long r = s_cu[0] + blockIdx.y * SLOT_T + tid; r < last; r += gridDim.y * SLOT_T) {
    int i = 0, slot = -1;
    while (s_cu[i + 1] <= r) ++i;
    const long long p = s_held[i] + (r - s_cu[i]);
    const long long j = p >> sh;
    if (j < W) {
      const int page = j >= s_have[i] ? pooled(s_start[i] + (j - s_have[i])) : a.table[(size_t)(b0 + i) * W + j];
      const long long at = (long long)page * T + (p & (T - 1));
      if (page >= 0 && at <= INT_MAX) slot = (int)at;
    }
    a.slots[r] = slot;
    a.positions[r] = (int)(p < INT_MAX ? p : INT_MAX);
  }
  // rows behind the last request's
  const long long w = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  for (long long r = s_all + w * SLOT_T + tid; r < a.n_rows; r += (long long)gridDim.x * gridDim.y * SLOT_T)
    a.slots[r] = a.positions[r] = -1;
}

// Many requests: sums of chunks of them, the sums before each chunk, then the requests and at last the rows, each by a
// launch of its own.  A chunk's two numbers (rows and lacking blocks, of it and then before it) wait between the
// launches in its first four entries of lens, which only its own workgroup writes.
constexpr int SLOT_CHUNK = 256, SLOT_SCAN_T = 1024;

struct SlotSums {
  long long rows, lack;
};
__device__ __forceinline__ SlotSums slot_sums_load(const int* p) {
  const unsigned a = p[0], b = p[1], c = p[2], d = p[3];
  return SlotSums{(long long)((unsigned long long)b << 32 | a), (long long)((unsigned long long)d << 32 | c)};
}
__device__ __forceinline__ void slot_sums_store(int* p, const SlotSums& s) {
  p[0] = (int)s.rows, p[1] = (int)(s.rows >> 32), p[2] = (int)s.lack, p[3] = (int)(s.lack >> 32);
}
// sums of the threads before this one, and of all; red: N / 64 entries
template <int N>
__device__ __forceinline__ SlotSums slot_scan(SlotSums x, SlotSums* red, SlotSums& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  SlotSums s = x;
  for (int o = 1; o < 64; o <<= 1) {
    const long long r = __shfl_up(s.rows, o), l = __shfl_up(s.lack, o);
    if (lane >= o) s.rows += r, s.lack += l;
  }
  if (lane == 63) red[wave] = s;
  __syncthreads();
  SlotSums before{s.rows - x.rows, s.lack - x.lack};
  all = SlotSums{0, 0};
  for (int w = 0; w < N / 64; ++w) {
    if (w < wave) before.rows += red[w].rows, before.lack += red[w].lack;
    all.rows += red[w].rows, all.lack += red[w].lack;
  }
  return before;
}
// a chunk's requests (the last takes the rest: every chunk has SLOT_CHUNK at least)
__device__ __forceinline__ int slot_chunk_end(const SlotArgs& a, int chunk, int chunks) {
  return chunk == chunks - 1 ? a.B : (chunk + 1) * SLOT_CHUNK;
}

__global__ __launch_bounds__(SLOT_T) void slots_sums_kernel(SlotArgs a) {
  __shared__ SlotSums red[SLOT_T / 64];
  const int b0 = blockIdx.x * SLOT_CHUNK, end = slot_chunk_end(a, blockIdx.x, gridDim.x), sh = __builtin_ctz(a.T);
  SlotSums s{0, 0}, all;
  for (int b = b0 + threadIdx.x; b < end; b += SLOT_T) {
    const long long h = max(a.held[b], 0), n = max(a.fresh[b], 0);
    s.rows += n;
    s.lack += slot_blocks(h + n, a.T, sh, a.width) - slot_blocks(h, a.T, sh, a.width);
  }
  slot_scan<SLOT_T>(s, red, all);
  if (threadIdx.x == 0) slot_sums_store(a.lens + b0, all);
}

__global__ __launch_bounds__(SLOT_SCAN_T) void slots_scan_kernel(SlotArgs a, int chunks) {
  __shared__ SlotSums red[SLOT_SCAN_T / 64];
  const int per = (chunks + SLOT_SCAN_T - 1) / SLOT_SCAN_T, c0 = threadIdx.x * per, end = min(c0 + per, chunks);
  SlotSums s{0, 0}, all;
  for (int c = c0; c < end; ++c) {
    const SlotSums x = slot_sums_load(a.lens + (size_t)c * SLOT_CHUNK);
    s.rows += x.rows, s.lack += x.lack;
  }
  SlotSums before = slot_scan<SLOT_SCAN_T>(s, red, all);
  for (int c = c0; c < end; ++c) {
    int* p = a.lens + (size_t)c * SLOT_CHUNK;
    const SlotSums x = slot_sums_load(p);
    slot_sums_store(p, before);
    before.rows += x.rows, before.lack += x.lack;
  }
  if (threadIdx.x == 0) {
    a.cu[0] = 0;
    a.used[0] = (int)min(all.lack, (long long)INT_MAX);
  }
}

__global__ __launch_bounds__(SLOT_T) void slots_requests_kernel(SlotArgs a) {
  constexpr int MOST = 2 * SLOT_CHUNK, PER = MOST / SLOT_T;  // requests of a chunk and of a thread
  __shared__ SlotSums red[SLOT_T / 64];
  __shared__ long long s_start[MOST + 1];
  __shared__ int s_have[MOST];
  const int tid = threadIdx.x, b0 = blockIdx.x * SLOT_CHUNK, nb = slot_chunk_end(a, blockIdx.x, gridDim.x) - b0;
  const int sh = __builtin_ctz(a.T), W = a.width;
  const SlotSums at = slot_sums_load(a.lens + b0);
  long long held[PER], fresh[PER];
  int have[PER], lack[PER];
  SlotSums s{0, 0}, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = tid * PER + i;
    held[i] = b < nb ? max(a.held[b0 + b], 0) : 0;
    fresh[i] = b < nb ? max(a.fresh[b0 + b], 0) : 0;
    have[i] = slot_blocks(held[i], a.T, sh, W);
    lack[i] = slot_blocks(held[i] + fresh[i], a.T, sh, W) - have[i];
    s.rows += fresh[i], s.lack += lack[i];
  }
  SlotSums before = slot_scan<SLOT_T>(s, red, all);  // (a barrier: everyone has read the chunk's sums)
  before.rows += at.rows, before.lack += at.lack;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = tid * PER + i;
    if (b < nb) {
      s_start[b] = before.lack;
      s_have[b] = have[i];
      before.rows += fresh[i], before.lack += lack[i];
      a.cu[b0 + b + 1] = (int)min(before.rows, (long long)INT_MAX);
      a.lens[b0 + b] = (int)min(held[i] + fresh[i], (long long)INT_MAX);
      if (b == nb - 1) s_start[nb] = before.lack;
    }
  }
  __syncthreads();
  // entries of the blocks taken here (an empty pool leaves -1)
  for (long long e = s_start[0] + tid; e < s_start[nb]; e += SLOT_T) {
    int lo = 0, hi = nb;  // the last request that starts at e or before
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_start[mid] <= e) lo = mid;
      else hi = mid;
    }
    a.table[(size_t)(b0 + lo) * W + s_have[lo] + (e - s_start[lo])] = e < a.n_pool ? a.pool[e] : -1;
  }
}

__global__ __launch_bounds__(SLOT_T) void slots_rows_kernel(SlotArgs a) {
  const int sh = __builtin_ctz(a.T);
  for (long long r = (long long)blockIdx.x * SLOT_T + threadIdx.x; r < a.n_rows; r += (long long)gridDim.x * SLOT_T) {
    int slot = -1, pos = -1, lo = 0, hi = a.B;  // the last request whose rows begin at r or before
    if (r < a.cu[a.B]) {
      while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (a.cu[mid] <= r) lo = mid;
        else hi = mid;
      }
      const long long p = (long long)max(a.held[lo], 0) + (r - a.cu[lo]), j = p >> sh;
      if (j < a.width) {
        const int page = a.table[(size_t)lo * a.width + j];
        const long long at = (long long)page * a.T + (p & (a.T - 1));
        if (page >= 0 && at <= INT_MAX) slot = (int)at;
      }
      pos = (int)min(p, (long long)INT_MAX);
    }
    a.slots[r] = slot;
    a.positions[r] = pos;
  }
}

void kvq_slots(const SlotArgs& a, hipStream_t st) {
  // Each workgroup of the single launch reads all lengths, a square of the requests in all.  us a call of single tokens, one
  // launch and four: 4096 requests 9.6 and 14.5, 8192 14.0 and 14.5, 16384 29 and 14.7, 131072 3510 and 18.6, 2^20 53 by four.
  if (a.B > SLOT_ALONE) {
    const int chunks = a.B / SLOT_CHUNK;
    hipLaunchKernelGGL(slots_sums_kernel, dim3(chunks), dim3(SLOT_T), 0, st, a);
    hipLaunchKernelGGL(slots_scan_kernel, dim3(1), dim3(SLOT_SCAN_T), 0, st, a, chunks);
    hipLaunchKernelGGL(slots_requests_kernel, dim3(chunks), dim3(SLOT_T), 0, st, a);
    if (a.n_rows)
      hipLaunchKernelGGL(slots_rows_kernel, dim3((unsigned)std::min(4096ll, ((long long)a.n_rows + SLOT_T - 1) / SLOT_T)), dim3(SLOT_T), 0, st, a);
    return;
  }
  // Workgroups for the same requests' rows: one for each 1024 of the rows that a group gets on average (a
  // prompt of 65536: 88 us with one, 4.6 with 64), and with many rows up to four for a group that gets more (one
  // such prompt among 2047 single tokens: 91 us with one, 31 with four, 26 with eight, which take
  // 0.9 us longer where all groups get the same).
  const int groups = (a.B + SLOT_SEQS - 1) / SLOT_SEQS;
  const int parts = std::max({1, std::min(256, a.n_rows / 1024 / groups), std::min(4, a.n_rows / 16384)});
  hipLaunchKernelGGL(slots_kernel, dim3(groups, parts), dim3(SLOT_T), 0, st, a);
}

// ---------------- rotary positions with several axes ----------------
// Pair j (elements j and j + half) of every head turns by
// pos[axis of j][t] * theta^(-j / half).  The angle is formed in float64 and
// reduced to a part of a half turn there, so far positions keep their phase;
// its remainder below the fp32 value enters to first order.  A workgroup makes
// the factors of its tokens' pairs once, in LDS, for all heads.  Bound by HBM
// at many tokens (each element read and written once): 16384 tokens of 32 + 8 heads of 128,
// 336 MB in 67 us a call, 5.0 TB/s, what a large copy reaches; by the launch at few (24
// fp32 tokens of 4 + 4 heads: 7.3 us a call, 3.2 the kernel).
constexpr int ROPE_T = 256;

template <typename E, int N>
struct alignas(sizeof(E) * N) RopeVec {
  E v[N];
};
__device__ __forceinline__ float rope_ld(float x) { return x; }
__device__ __forceinline__ float rope_ld(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void rope_st(float& d, float x) { d = x; }
// one rounding to bf16, of the finished value (NaN kept: the carry of the rounding must not make it infinite)
__device__ __forceinline__ void rope_st(uint16_t& d, float x) {
  const uint32_t u = __float_as_uint(x);
  d = x == x ? (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16) : (uint16_t)((u >> 16) | 0x40u);
}

template <typename E, int N>
__global__ __launch_bounds__(ROPE_T) void rope_axes_kernel(RopeArgs a, int TB) {
  extern __shared__ float2 fac[];  // [TB][half]
  const int tid = threadIdx.x, half = a.half, t0 = blockIdx.x * TB, nt = min(TB, a.T - t0);
  for (int i = tid; i < nt * half; i += ROPE_T) {
    const int t = i / half, j = i - t * half;
    int ax = 0, end = a.section[0];
    while (j >= end) end += a.section[++ax];
    // angle / pi, less whole turns: in [-1, 1]
    const double turn = (double)a.pos[(size_t)ax * a.T + t0 + t] * (exp2(-(double)j / half * a.log2_theta) * 0.15915494309189535);
    const double x = 2.0 * (turn - rint(turn));
    const float xh = (float)x;
    const float d = (float)(x - (double)xh) * 3.14159265f;
    float s, c;
    sincospif(xh, &s, &c);
    fac[i] = make_float2(fmaf(-s, d, c), fmaf(c, d, s));
  }
  __syncthreads();
  const int pairs = half / N, rest = (a.D - 2 * half) / N, per = pairs + rest, heads = a.Hq + a.Hkv;
  typedef RopeVec<E, N> V;
  for (int i = tid; i < nt * heads * per; i += ROPE_T) {
    const int t = i / (heads * per), r = i - t * heads * per, h = r / per, c = r - h * per;
    const size_t tok = t0 + t;
    const E* src = h < a.Hq ? (const E*)a.q + tok * a.ld_q + (size_t)h * a.D
                            : (const E*)a.k + tok * a.ld_k + (size_t)(h - a.Hq) * a.D;
    E* dst = h < a.Hq ? (E*)a.qo + tok * a.ld_qo + (size_t)h * a.D
                      : (E*)a.ko + tok * a.ld_ko + (size_t)(h - a.Hq) * a.D;
    if (c < pairs) {
      const V x = *(const V*)(src + c * N), y = *(const V*)(src + half + c * N);
      V u, w;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 f = fac[t * half + c * N + e];
        const float p = rope_ld(x.v[e]), q = rope_ld(y.v[e]);
        rope_st(u.v[e], p * f.x - q * f.y);
        rope_st(w.v[e], q * f.x + p * f.y);
      }
      *(V*)(dst + c * N) = u;
      *(V*)(dst + half + c * N) = w;
    } else {
      const int o = 2 * half + (c - pairs) * N;
      *(V*)(dst + o) = *(const V*)(src + o);
    }
  }
}

void rope_axes(const RopeArgs& a, hipStream_t st) {
  // tokens a workgroup: 12 KB of factors at most (fewer tokens would make 2^25 of them more threads than a launch takes)
  const int TB = std::max(3, std::min(4, 1024 / a.half));
  const dim3 grid((a.T + TB - 1) / TB);
  const size_t lds = (size_t)TB * a.half * sizeof(float2);
  // 16-byte accesses where every row, head and half starts on one (the 16384 tokens above: 64 us, 150 by elements)
  const int N = a.bf16 ? 8 : 4;
  const uintptr_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.qo | (uintptr_t)a.ko;
  const bool vec = at % 16 == 0 && a.half % N == 0 && a.D % N == 0 &&
                   (a.ld_q | a.ld_k | a.ld_qo | a.ld_ko) % N == 0;
  if (a.bf16) {
    if (vec) hipLaunchKernelGGL((rope_axes_kernel<uint16_t, 8>), grid, dim3(ROPE_T), lds, st, a, TB);
    else hipLaunchKernelGGL((rope_axes_kernel<uint16_t, 1>), grid, dim3(ROPE_T), lds, st, a, TB);
  } else {
    if (vec) hipLaunchKernelGGL((rope_axes_kernel<float, 4>), grid, dim3(ROPE_T), lds, st, a, TB);
    else hipLaunchKernelGGL((rope_axes_kernel<float, 1>), grid, dim3(ROPE_T), lds, st, a, TB);
  }
}

// the same factors as a session's table, one thread a pair (the float64 formula of rope_table, whose
// bits equal positions reproduce)
__global__ __launch_bounds__(256) void rope_axes_table_kernel(RopeTableArgs a) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)a.n * a.half) return;
  const int p = (int)(i / a.half), j = (int)(i - (size_t)p * a.half);
  int ax = 0, end = a.section[0];
  while (j >= end) end += a.section[++ax];
  const double ang = (double)a.pos[(size_t)ax * a.n + p] * pow(a.theta, -(double)j / a.half);
  a.tab[i] = make_float2((float)cos(ang), (float)sin(ang));
}

void rope_axes_table(const RopeTableArgs& a, hipStream_t st) {
  const size_t n = (size_t)a.n * a.half;
  hipLaunchKernelGGL(rope_axes_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a);
}

// ---------------- a session's cache as rows ----------------
// One thread copies eight dims of one position and head: 16 bytes of a key tile, and the value
// tiles' elements one by one.  VEC: the outputs start on 16 bytes, else they are written by elements.
template <bool VEC>
__global__ __launch_bounds__(256) void read_kv_bf16_kernel(int B, int n, int Hkv, int D, int Lmax, const uint16_t* kc,
                                                           const uint16_t* vc, uint16_t* k, uint16_t* v) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const int per = D / 8;
  if (i >= (size_t)B * n * Hkv * per) return;
  const int c = (int)(i % per), h = (int)(i / per % Hkv), p = (int)(i / ((size_t)per * Hkv) % n);
  const size_t b = i / ((size_t)per * Hkv * n), base = (b * Hkv + h) * (size_t)Lmax * D;
  RopeVec<uint16_t, 8> x, y;
  x = *(const RopeVec<uint16_t, 8>*)(kc + base + tile16x32_index(p, c * 8, D));
#pragma unroll
  for (int e = 0; e < 8; ++e) y.v[e] = vc[base + vtile_index(c * 8 + e, p, Lmax)];
  if constexpr (VEC) {
    *(RopeVec<uint16_t, 8>*)(k + i * 8) = x;
    *(RopeVec<uint16_t, 8>*)(v + i * 8) = y;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) k[i * 8 + e] = x.v[e], v[i * 8 + e] = y.v[e];
  }
}
__global__ __launch_bounds__(256) void read_kv_f32_kernel(int B, int n, int Hkv, int D, int Lmax, const float* kc, const float* vc,
                                                          float* k, float* v) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (size_t)B * n * Hkv * D) return;
  const int d = (int)(i % D), h = (int)(i / D % Hkv), p = (int)(i / ((size_t)D * Hkv) % n);
  const size_t b = i / ((size_t)D * Hkv * n), base = (b * Hkv + h) * (size_t)Lmax * D;
  k[i] = kc[base + (size_t)p * D + d];
  v[i] = vc[base + (size_t)d * Lmax + p];
}

void read_kv(const Dims& dm, int B, int n, int Lmax, const void* kc, const void* vc, void* k, void* v, hipStream_t st) {
  const size_t all = (size_t)B * n * dm.Hkv * dm.D;
  const bool vec = (((uintptr_t)k | (uintptr_t)v) & 15) == 0;
  if (dm.bf16)
    hipLaunchKernelGGL(vec ? read_kv_bf16_kernel<true> : read_kv_bf16_kernel<false>, dim3((unsigned)((all / 8 + 255) / 256)), dim3(256),
                       0, st, B, n, dm.Hkv, dm.D, Lmax, (const uint16_t*)kc, (const uint16_t*)vc, (uint16_t*)k, (uint16_t*)v);
  else
    hipLaunchKernelGGL(read_kv_f32_kernel, dim3((unsigned)((all + 255) / 256)), dim3(256), 0, st, B, n, dm.Hkv, dm.D, Lmax,
                       (const float*)kc, (const float*)vc, (float*)k, (float*)v);
}

}  // namespace ssd
