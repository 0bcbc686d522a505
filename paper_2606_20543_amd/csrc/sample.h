// Sampling of given logits with temperature, top-k, top-p and min-p from given
// uniforms (included by kernels_misc.hip).
//
// A code's weight is w = exp((l - max) / T), in float64, held as the integer
// nearest to 2^45 w: sums of integers are the same in any order, so the result
// does not depend on which atomic came first, and a weight that vanishes there
// (below 2^-46 of the largest) is never drawn.  The codes that the three
// settings keep are a prefix of the order (logit descending, code ascending):
// the first top_k of it, the shortest prefix of those that holds top_p of
// their mass, and the weights of at least min_p (of the largest weight).  So
// one pair (logit, code) bounds the set.  It is found without a sort: the
// codes are counted (top-k) and their weights summed (top-p) in 2048 bins of
// equal width over the logits that have a weight, and the few codes of the bin
// that a bound falls into are ranked against each other; a bin of more is
// divided again.  The draw is the smallest kept code whose running sum (code
// order) exceeds u times the total.  One workgroup of 16 waves a row, the row
// in registers up to 32768 codes.
//
// Four rows of 16384 codes with top-k and top-p: 20.5 us a call, a chain of some fifteen
// barriers in one workgroup each.  512 rows of 32768, settings of their own: 76 us (67 MB, 13 us
// at the rate of a large copy; two rows a CU one after the other).  With the same settings in all rows:
// reading and the draw 37, a top-k 21 more, a top-p 26, both 39: atomics on shared memory, one
// or two a code at about a lane and cycle, and the float64 exponentials.  Rows that start on
// 16 bytes are read by four codes (17 us less).
#pragma once

namespace ssd {

constexpr int LS_T = 1024, LS_W = LS_T / 64;
constexpr int LS_BINS = 2 * LS_T, LS_LIST = 1024;
constexpr double LS_ONE = 35184372088832.0;  // 2^45
constexpr int LS_POW_LOG2 = 8, LS_POW = 1 << LS_POW_LOG2;

struct LsShared {
  unsigned cnt[LS_BINS];
  unsigned long long wgt[LS_BINS];
  // codes of the bin that a bound falls into: logit, code, weight, and how many and how much come before
  float lv[LS_LIST];
  int li[LS_LIST];
  unsigned long long lw[LS_LIST];
  unsigned lc[LS_LIST];
  unsigned long long lb[LS_LIST];
  double pow2[LS_POW];  // 2^(45 + i / 256)
  unsigned long long wred[LS_W];
  unsigned cred[LS_W];
  float fmn[LS_W], fmx[LS_W];
  int ired[LS_W];
  int n, bin;
  unsigned c0;
  unsigned long long w0;
  float bv;
  int bi;
};

// Sums and extrema over lanes by moves between lanes of a row of 16 (no trip through shared memory);
// every lane of the wave takes part.
template <int CTRL, int ROWS = 15>
__device__ __forceinline__ unsigned ls_move(unsigned v) {  // 0 where no lane gives one
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 15, false);
}
template <int CTRL, int ROWS = 15>
__device__ __forceinline__ float ls_move(float v) {
  return __uint_as_float(ls_move<CTRL, ROWS>(__float_as_uint(v)));
}
template <int CTRL, int ROWS = 15>
__device__ __forceinline__ unsigned long long ls_move(unsigned long long v) {
  return (unsigned long long)ls_move<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | ls_move<CTRL, ROWS>((unsigned)v);
}
constexpr int LS_ROR = 0x120, LS_SHR = 0x110, LS_BCAST15 = 0x142, LS_BCAST31 = 0x143;
// op over each row's lanes, in all of them
template <typename T, typename Op>
__device__ __forceinline__ T ls_row(T v, Op op) {
  v = op(v, ls_move<LS_ROR + 8>(v));
  v = op(v, ls_move<LS_ROR + 4>(v));
  v = op(v, ls_move<LS_ROR + 2>(v));
  return op(v, ls_move<LS_ROR + 1>(v));
}
template <typename T, typename Op>
__device__ __forceinline__ T ls_wave(T v, Op op) {
  v = ls_row(v, op);
  v = op(v, __shfl_xor(v, 16));
  return op(v, __shfl_xor(v, 32));
}
// sums of the lanes up to each
template <typename T>
__device__ __forceinline__ T ls_scan(T v) {
  v += ls_move<LS_SHR + 1>(v);
  v += ls_move<LS_SHR + 2>(v);
  v += ls_move<LS_SHR + 4>(v);
  v += ls_move<LS_SHR + 8>(v);
  v += ls_move<LS_BCAST15, 10>(v);         // into the odd rows
  return v + ls_move<LS_BCAST31, 12>(v);   // into the upper half
}
struct LsAdd {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct LsMax {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct LsMin {
  __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
};
// over the waves' entries: the sum of those before the wave, of all
static_assert(LS_W == 16, "a row of lanes");
template <typename T>
__device__ __forceinline__ T ls_before(const T* red, int lane, int wave) {
  const T x = red[lane & 15];
  return ls_row((lane & 15) < wave ? x : T(0), LsAdd{});
}
template <typename T>
__device__ __forceinline__ T ls_all(const T* red, int lane) {
  return ls_row(red[lane & 15], LsAdd{});
}

// a logit as it counts: NaN is never drawn, +inf is the largest finite number
__device__ __forceinline__ float ls_clean(float l) { return l == l ? fminf(l, 3.4028234664e38f) : -INFINITY; }

// The codes of a wave, in groups of 256 (four a lane), wave w the w-th contiguous segment of the
// row; -inf past its end.  NG > 0: held in registers, else read by every pass.
template <int NG>
struct LsRow {
  const float* row;
  int V, beg, groups;
  bool vec;
  mutable float4 held[NG > 0 ? NG : 1];
  __device__ __forceinline__ LsRow(const float* r, int v) : row(r), V(v) {
    const int all = (V + 255) / 256, per = (all + LS_W - 1) / LS_W, w = threadIdx.x >> 6;
    beg = w * per * 256 + (threadIdx.x & 63) * 4;
    groups = max(0, min(per, all - w * per));
    vec = (V & 3) == 0 && (((uintptr_t)row) & 15) == 0;
    if constexpr (NG > 0) {
#pragma unroll
      for (int i = 0; i < NG; ++i) held[i] = i < groups ? read(i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    }
  }
  __device__ __forceinline__ float4 read(int i) const {
    const int v = beg + i * 256;
    float4 f = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (vec) {
      if (v < V) f = *(const float4*)(row + v);
    } else {
      if (v < V) f.x = row[v];
      if (v + 1 < V) f.y = row[v + 1];
      if (v + 2 < V) f.z = row[v + 2];
      if (v + 3 < V) f.w = row[v + 3];
    }
    return make_float4(ls_clean(f.x), ls_clean(f.y), ls_clean(f.z), ls_clean(f.w));
  }
  // fn(first code of the lane, its four logits) over the groups in order, every lane together
  template <typename F>
  __device__ __forceinline__ void each(F fn) const {
    if constexpr (NG > 0) {
#pragma unroll
      for (int i = 0; i < NG; ++i)
        if (i < groups) {
          // (values that the compiler takes for new ones: what a pass computes of them is computed in that
          // pass, not ahead of the barriers before it nor kept from an earlier one, which ends in scratch memory.  Of
          // eight groups ten registers still do, 44 bytes a lane; of four none.)
          asm volatile("" : "+v"(held[i].x), "+v"(held[i].y), "+v"(held[i].z), "+v"(held[i].w));
          const float x[4] = {held[i].x, held[i].y, held[i].z, held[i].w};
          fn(beg + i * 256, x);
        }
    } else {
      again(fn);
    }
  }
  // the same, read from memory: for what few rows do (unrolled over held values it would take registers from all)
  template <typename F>
  __device__ __forceinline__ void again(F fn) const {
#pragma unroll 2
    for (int i = 0; i < groups; ++i) {
      const float4 f = read(i);
      const float x[4] = {f.x, f.y, f.z, f.w};
      fn(beg + i * 256, x);
    }
  }
};

// 2^45 exp((l - mx) / T) for logits that have a weight: y = 256 (l - mx) / (T ln 2) is split into a whole
// number n (the low bits of 1.5 2^52 + y), whose power of two is a table entry with n / 256 added to its
// exponent, and a rest f, |f| <= 1/2, whose power 2^(f / 256) is a polynomial of degree 4 (off by 2^-54).
// (A table of 1024 and degree 3 measured the same.)
struct LsWeight {
  float mx;
  double scale;  // 256 / (T ln 2)
  const double* pow2;
  __device__ __forceinline__ double operator()(float l) const {
    constexpr double MAGIC = 6755399441055744.0, C = 0.6931471805599453 / LS_POW;
    const double y = ((double)l - (double)mx) * scale, t = y + MAGIC, f = y - (t - MAGIC);
    const int n = (int)(unsigned)__double_as_longlong(t);
    const double p = fma(f, fma(f, fma(f, fma(f, C * C * C * C / 24, C * C * C / 6), C * C / 2), C), 1.0);
    const long long e = (long long)((unsigned long long)(unsigned)((n >> LS_POW_LOG2) << 20) << 32);
    return p * __longlong_as_double(__double_as_longlong(pow2[n & (LS_POW - 1)]) + e);
  }
  // the nearest integer to w <= 2^45, as a double (a thread's sums stay exact), and from the low bits of 2^52 + w
  static __device__ __forceinline__ double whole(double w) { return (w + 4503599627370496.0) - 4503599627370496.0; }
  static __device__ __forceinline__ unsigned long long fix(double w) {
    return (unsigned long long)__double_as_longlong(w + 4503599627370496.0) - 0x4330000000000000ull;
  }
};

// what the bound is asked to reach: so many codes, or so much mass
struct LsGoal {
  bool by_weight;
  unsigned count;
  double mass;
  __device__ __forceinline__ bool operator()(unsigned long long c, unsigned long long w) const {
    return by_weight ? (double)w >= mass : c >= count;
  }
};

// equal-width bins over [lo, hi], the first the largest logits: a monotone map (products,
// subtraction and truncation are); the factor k, a power of two, keeps the width a normal number,
// so that lo and hi never share a bin
struct LsBins {
  float lo, hi, k, sc;
  __device__ __forceinline__ LsBins(float l, float h) : lo(l), hi(h) {
    k = hi - lo > 1e38f ? 0.25f : hi - lo < 1e-30f ? 0x1p100f : 1.f;
    const float width = hi * k - lo * k;
    sc = width > 0.f ? (float)LS_BINS / width : 0.f;
  }
  __device__ __forceinline__ bool in(float l) const { return l >= lo && l <= hi; }
  __device__ __forceinline__ int operator()(float l) const { return min(LS_BINS - 1, (int)((hi * k - l * k) * sc)); }
};

// codes and mass up to this thread's two bins (with what lies before the bins), and the bins' own
struct LsCumul {
  unsigned ca, cb;
  unsigned long long wa, wb, c, w;  // c, w: through the second bin
};

template <int NG>
__device__ __forceinline__ LsCumul ls_histogram(const LsRow<NG>& row, const LsWeight& wt, const LsBins& bins, bool count, bool weigh,
                                                unsigned c0, unsigned long long w0, LsShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  static_assert(LS_BINS == 2 * LS_T, "two bins a thread");
  sh.cnt[2 * tid] = sh.cnt[2 * tid + 1] = 0;
  sh.wgt[2 * tid] = sh.wgt[2 * tid + 1] = 0;
  __syncthreads();
  row.each([&](int, const float(&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (bins.in(x[e])) {
        const int b = bins(x[e]);
        if (count) atomicAdd(&sh.cnt[b], 1u);
        if (weigh) atomicAdd(&sh.wgt[b], LsWeight::fix(wt(x[e])));
      }
  });
  __syncthreads();
  LsCumul q;
  q.ca = sh.cnt[2 * tid], q.cb = sh.cnt[2 * tid + 1];
  q.wa = sh.wgt[2 * tid], q.wb = sh.wgt[2 * tid + 1];
  q.c = ls_scan(q.ca + q.cb);
  q.w = weigh ? ls_scan(q.wa + q.wb) : 0;
  if (lane == 63) {
    sh.cred[wave] = (unsigned)q.c;
    sh.wred[wave] = q.w;
  }
  __syncthreads();
  q.c += c0 + ls_before(sh.cred, lane, wave);
  q.w += w0 + ls_before(sh.wred, lane, wave);
  return q;
}

// The shortest prefix of the order that reaches the goal, given the histogram of the logits in bins
// (divided further where a bin holds too many): its bound in sh.bv, sh.bi, its codes and mass
// in sh.c0, sh.w0.  All codes in the bins fall short: bv = bins.lo, bi = INT_MAX.
template <int NG>
__device__ __forceinline__ void ls_bound(const LsRow<NG>& row, const LsWeight& wt, LsBins bins, LsCumul q, const LsGoal& goal, bool weigh,
                                      LsShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  while (true) {
    __syncthreads();
    if (tid == 0) {
      sh.n = 0;
      sh.bin = LS_BINS;
    }
    __syncthreads();
    const uint64_t there = __ballot(goal(q.c, q.w));
    if (there && lane == __builtin_ctzll(there)) atomicMin(&sh.bin, goal(q.c - q.cb, q.w - q.wb) ? 2 * tid : 2 * tid + 1);
    __syncthreads();
    const int bin = sh.bin;
    if (bin == LS_BINS) {  // everything is kept
      if (tid == LS_T - 1) {
        sh.c0 = (unsigned)q.c;
        sh.w0 = q.w;
        sh.bv = bins.lo;
        sh.bi = 0x7fffffff;
      }
      __syncthreads();
      return;
    }
    if (bin >> 1 == tid) {  // what lies before the bin
      sh.c0 = (unsigned)(q.c - q.cb - (bin & 1 ? 0 : q.ca));
      sh.w0 = q.w - q.wb - (bin & 1 ? 0 : q.wa);
    }
    // the bin's codes: a list, and the range of their logits
    float mn = INFINITY, mx = -INFINITY;
    row.each([&](int v, const float(&x)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (bins.in(x[e]) && bins(x[e]) == bin) {
          mn = fminf(mn, x[e]);
          mx = fmaxf(mx, x[e]);
          const int at = atomicAdd(&sh.n, 1);
          if (at < LS_LIST) {
            sh.lv[at] = x[e];
            sh.li[at] = v + e;
          }
        }
    });
    mn = ls_wave(mn, LsMin{});
    mx = ls_wave(mx, LsMax{});
    if (lane == 0) {
      sh.fmn[wave] = mn;
      sh.fmx[wave] = mx;
    }
    __syncthreads();
    const int n = sh.n;
    const unsigned c0 = sh.c0;
    const unsigned long long w0 = sh.w0;
    if (n <= LS_LIST) {
      // rank the list: `parts` threads share a code's comparisons
      if (tid < n) {
        sh.lw[tid] = weigh ? LsWeight::fix(wt(sh.lv[tid])) : 0;
        sh.lc[tid] = 0;
        sh.lb[tid] = 0;
      }
      __syncthreads();
      const int pad = n > 1 ? 1 << (32 - __builtin_clz(n - 1)) : 1, parts = LS_T / pad, i = tid & (pad - 1);
      if (i < n) {
        const float li = sh.lv[i];
        const int ii = sh.li[i];
        unsigned c = 0;
        unsigned long long w = 0;
        for (int j = tid / pad; j < n; j += parts) {
          const float lj = sh.lv[j];
          if (lj > li || (lj == li && sh.li[j] < ii)) {
            ++c;
            w += sh.lw[j];
          }
        }
        atomicAdd(&sh.lc[i], c);
        atomicAdd(&sh.lb[i], w);
      }
      __syncthreads();
      // the one code with the bound inside it
      if (tid < n) {
        const unsigned c = c0 + sh.lc[tid];
        const unsigned long long w = w0 + sh.lb[tid];
        if (!goal(c, w) && goal(c + 1, w + sh.lw[tid])) {
          sh.bv = sh.lv[tid];
          sh.bi = sh.li[tid];
          sh.c0 = c + 1;
          sh.w0 = w + sh.lw[tid];
        }
      }
      __syncthreads();
      return;
    }
    mn = ls_row(sh.fmn[lane & 15], LsMin{});
    mx = ls_row(sh.fmx[lane & 15], LsMax{});
    if (mn == mx) {
      // equal logits: so many of them, in code order
      const unsigned long long w1 = weigh ? LsWeight::fix(wt(mx)) : 0;
      unsigned take = goal.count - c0;
      if (goal.by_weight) take = w1 ? max((unsigned)fmin(ceil((goal.mass - (double)w0) / (double)w1), (double)n), 1u) : (unsigned)n;
      unsigned mine = 0;  // ties of this wave's segment, then those before it
      row.again([&](int, const float(&x)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) mine += __popcll(__ballot(x[e] == mx));
      });
      __syncthreads();
      if (lane == 0) sh.cred[wave] = mine;
      __syncthreads();
      unsigned at = ls_before(sh.cred, lane, wave);
      row.again([&](int v, const float(&x)[4]) {
        unsigned k = at, all = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint64_t m = __ballot(x[e] == mx);
          k += __popcll(m & ((1ull << lane) - 1));
          all += __popcll(m);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (x[e] == mx && k++ == take - 1) sh.bi = v + e;
        at += all;
      });
      if (tid == 0) {
        sh.bv = mx;
        sh.c0 = c0 + take;
        sh.w0 = w0 + take * w1;
      }
      __syncthreads();
      return;
    }
    bins = LsBins(mn, mx);
    __syncthreads();  // (everyone has read c0, w0 and the ranges)
    q = ls_histogram(row, wt, bins, !goal.by_weight, weigh, c0, w0, sh);
  }
}

template <int NG>
__global__ __launch_bounds__(LS_T) void sample_logits_kernel(SampleArgs a) {
  __shared__ LsShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x, V = a.V;
  const double T = a.temperatures ? (double)a.temperatures[r] : a.temperature;
  const int top_k = a.top_ks ? a.top_ks[r] : a.top_k;
  const double top_p = a.top_ps ? (double)a.top_ps[r] : a.top_p;
  const double min_any = a.min_ps ? (double)a.min_ps[r] : a.min_p;
  const double min_p = min_any > 1.0 ? 1.0 : min_any;  // the largest always stays (NaN: nothing is below it)
  const double u = a.u[r];
  const LsRow<NG> row(a.logits + (size_t)r * a.ld, V);
  if (tid < LS_POW) sh.pow2[tid] = LS_ONE * exp2((double)tid / LS_POW);
  float mx = -INFINITY, mn = INFINITY;  // (the least that can be drawn)
  row.each([&](int, const float(&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mx = fmaxf(mx, x[e]);
      mn = fminf(mn, x[e] == -INFINITY ? INFINITY : x[e]);
    }
  });
  mx = ls_wave(mx, LsMax{});
  mn = ls_wave(mn, LsMin{});
  if (lane == 0) {
    sh.fmx[wave] = mx;
    sh.fmn[wave] = mn;
  }
  __syncthreads();
  mx = ls_row(sh.fmx[lane & 15], LsMax{});
  mn = ls_row(sh.fmn[lane & 15], LsMin{});
  if (mx == -INFINITY || !(T > 0.0)) {  // nothing to draw, or the largest (its lowest code)
    int am = 0x7fffffff;
    row.again([&](int v, const float(&x)[4]) {
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (x[e] == mx) am = min(am, v + e);
    });
    for (int o = 32; o > 0; o >>= 1) am = min(am, __shfl_xor(am, o));
    if (lane == 0) sh.ired[wave] = am;
    __syncthreads();
    if (tid == 0) {
      for (int x = 1; x < LS_W; ++x) am = min(am, sh.ired[x]);
      a.tokens[r] = mx == -INFINITY ? -1 : am + a.add;
      if (a.probs) a.probs[r] = mx == -INFINITY ? 0.f : 1.f;
    }
    return;
  }
  const LsWeight wt{mx, fmin(LS_POW / (T * 0.6931471805599453), 1e300), sh.pow2};
  const double min_w = min_p * LS_ONE;
  // logits below this have no weight (32 > 46 ln 2)
  const float floor_l = fmaxf((float)((double)mx - 32.0 * T), -3.4028234664e38f);
  float bv = floor_l;
  int bi = 0x7fffffff;
  const bool by_k = top_k > 0 && top_k < V, by_p = top_p < 1.0;
  if (by_k || by_p) {
    const LsBins bins(fmaxf(floor_l, mn), mx);  // (from floor_l alone: 88 us in place of 76, warm rows share few bins)
    const LsCumul q = ls_histogram(row, wt, bins, by_k, by_p, 0u, 0ull, sh);
    double mass = 0.0;
    if (by_k) {
      ls_bound(row, wt, bins, q, LsGoal{false, (unsigned)top_k, 0.0}, by_p, sh);
      bv = sh.bv;
      bi = sh.bi;
      mass = (double)sh.w0;
    } else {
      mass = (double)ls_all(sh.wred, lane);
    }
    if (by_p) {  // (with a top-k the prefix ends inside that of the top-k)
      ls_bound(row, wt, bins, q, LsGoal{true, 0u, fmax(top_p * mass, 1.0)}, true, sh);
      bv = sh.bv;
      bi = sh.bi;
    }
    __syncthreads();
  }
  // The draw: the sums of the kept weights by wave and group (256 codes), the wave and the group
  // whose running sum passes the target, and there the lane and the code.
  auto kept = [&](float l, int v) { return l > bv || (l == bv && v <= bi); };
  auto weight = [&](float l) {  // whole, 0 below min_p
    const double w = wt(l);
    return w < min_w ? 0.0 : LsWeight::whole(w);
  };
  auto group_sum = [&](int v, const float(&x)[4], double (&w)[4]) {
    bool k[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = kept(x[e], v + e);
      w[e] = 0.0;
    }
    if (__any(k[0] || k[1] || k[2] || k[3])) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double y = weight(k[e] ? x[e] : bv);
        w[e] = k[e] ? y : 0.0;
      }
    }
    return (w[0] + w[1]) + (w[2] + w[3]);
  };
  double gs[NG > 0 ? NG : 1], s = 0.0;
  {
    int i = 0;
#pragma unroll
    for (int g = 0; g < (NG > 0 ? NG : 1); ++g) gs[g] = 0.0;
    row.each([&](int v, const float(&x)[4]) {
      double w[4];
      const double t = group_sum(v, x, w);
      s += t;
      if constexpr (NG > 0) gs[i++] = t;
    });
  }
  const unsigned long long inc = ls_scan((unsigned long long)s);
  if (lane == 63) sh.wred[wave] = inc;
  if (tid == 0) sh.bi = 0x7fffffff;
  __syncthreads();
  const unsigned long long total = ls_all(sh.wred, lane), base = ls_before(sh.wred, lane, wave);
  const double target = (u > 0.0 ? u : 0.0) * (double)total;
  auto draw = [&](int v, float l) {
    a.tokens[r] = v + a.add;
    if (a.probs) a.probs[r] = (float)(wt(l) / (double)total);
    sh.bi = v;
  };
  if (!((double)base > target) && (double)(base + __shfl(inc, 63)) > target) {
    unsigned long long run = base;
    int at = 0;
    bool found = false;
    auto pass = [&](double lanes) {  // a group's sum
      const unsigned long long t = ls_wave((unsigned long long)lanes, LsAdd{});
      found |= (double)(run + t) > target;
      run += found ? 0 : t;
      at += found ? 0 : 1;
    };
    if constexpr (NG > 0) {
#pragma unroll
      for (int g = 0; g < NG; ++g) pass(gs[g]);
    } else {
      row.each([&](int v, const float(&x)[4]) {
        if (found) return;
        double w[4];
        pass(group_sum(v, x, w));
      });
    }
    const float4 f = row.read(at);
    const float x[4] = {f.x, f.y, f.z, f.w};
    const int v = row.beg + at * 256;
    double w[4];
    const unsigned long long t = (unsigned long long)group_sum(v, x, w);
    unsigned long long c = run + (ls_scan(t) - t);
    if (!((double)c > target) && (double)(c + t) > target) {
      found = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c += (unsigned long long)w[e];
        if (!found && (double)c > target) {
          found = true;
          draw(v + e, x[e]);
        }
      }
    }
  }
  __syncthreads();
  if (sh.bi == 0x7fffffff) {  // u at or past one: the last code that has a weight
    int last = -1;
    row.again([&](int v, const float(&x)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (kept(x[e], v + e) && weight(x[e]) > 0.0) last = max(last, v + e);
    });
    for (int o = 32; o > 0; o >>= 1) last = max(last, __shfl_xor(last, o));
    if (lane == 0) sh.ired[wave] = last;
    __syncthreads();
    if (tid == 0) {
      for (int x = 0; x < LS_W; ++x) last = max(last, sh.ired[x]);
      draw(last, ls_clean(a.logits[(size_t)r * a.ld + last]));
    }
  }
}

void sample_logits(const SampleArgs& a, hipStream_t st) {
  // the longest row that is held: 4 codes a thread and group (4 groups take fewer registers: 256 rows of 16384
  // 22 us; rows past 8 groups are read again from the caches by every pass)
  if (a.V <= 4 * 4 * LS_T)
    hipLaunchKernelGGL(sample_logits_kernel<4>, dim3(a.R), dim3(LS_T), 0, st, a);
  else if (a.V <= 8 * 4 * LS_T)
    hipLaunchKernelGGL(sample_logits_kernel<8>, dim3(a.R), dim3(LS_T), 0, st, a);
  else
    hipLaunchKernelGGL(sample_logits_kernel<0>, dim3(a.R), dim3(LS_T), 0, st, a);
}

}  // namespace ssd
