// Sampling of given logits with temperature, top-k, top-p and min-p from given
// uniforms (included by kernels_misc.hip, whose row segments it uses).
//
// A code's weight is w = exp((l - max) / T), in float64, held as the integer
// nearest to 2^45 w: sums of integers are the same in any order, so the result
// does not depend on which atomic came first, and a weight that vanishes there
// (below 2^-46 of the largest) is never drawn.  The codes that the three
// settings keep are a prefix of the order (logit descending, code ascending):
// the first top_k of it, the shortest prefix of those that holds top_p of
// their mass, and the weights of at least min_p (of the largest weight).  So
// one pair (logit, code) bounds the set.  It is found without a sort: the
// codes are counted and their weights summed in 2048 bins of equal width over
// the logits that have a weight, the bin that the bound falls into is narrowed
// the same way until it holds few codes, and those are ranked against each other.
// The draw is the smallest kept code whose running sum (code order) exceeds
// u times the total.  One workgroup of 16 waves a row.
#pragma once

namespace ssd {

constexpr int LS_BINS = 2048, LS_LIST = 1024;
constexpr double LS_ONE = 35184372088832.0;  // 2^45

struct LsShared {
  unsigned cnt[LS_BINS];
  unsigned long long wgt[LS_BINS];
  float lv[LS_LIST];
  int li[LS_LIST];
  unsigned long long lw[LS_LIST];
  unsigned lc[LS_LIST];            // codes before, weight before
  unsigned long long lb[LS_LIST];
  unsigned long long wred[SMP_W], wred2[SMP_W];
  unsigned cred[SMP_W];
  float fmn[SMP_W], fmx[SMP_W];
  int ired[SMP_W];
  int n, bin;
  unsigned c0;
  unsigned long long w0;
  float bv;
  int bi;
};

__device__ __forceinline__ unsigned long long ls_scan(unsigned long long v, int lane) {
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}

template <int NG>
struct LsRow {
  const Seg<NG>& g;
  float mx;
  double inv;  // 1 / T
  __device__ __forceinline__ LsRow(const Seg<NG>& s, float m, double i) : g(s), mx(m), inv(i) {}
  __device__ __forceinline__ double w(float l) const { return exp(((double)l - (double)mx) * inv); }
  __device__ __forceinline__ unsigned long long fix(double x) const { return (unsigned long long)(x * LS_ONE + 0.5); }
};

// a logit as it counts: NaN is never drawn, +inf is the largest finite number
__device__ __forceinline__ float ls_clean(float l) { return l == l ? fminf(l, 3.4028234664e38f) : -INFINITY; }

// Shortest prefix of the order with at least `need_c` codes, or with a mass of at least
// need_w (by_weight), among the codes of a logit >= floor_l; the bound is left in
// sh.bv, sh.bi, the prefix's codes and mass in sh.c0, sh.w0.  All codes fall short: bv = floor_l, bi = INT_MAX.
template <int NG>
__device__ void ls_bound(const LsRow<NG>& r, float floor_l, bool by_weight, unsigned need_c, double need_w, LsShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float hi = r.mx, lo = floor_l;  // the codes still to be told apart have lo <= l <= hi
  unsigned c0 = 0;                // codes above hi, and their mass
  unsigned long long w0 = 0;
  while (true) {
    // bins of equal width, the first the largest logits (a monotone map: products,
    // subtraction and truncation are; the factor k, a power of two, keeps the width a
    // normal number, so that lo and hi never share a bin)
    const float k = hi - lo > 1e38f ? 0.25f : hi - lo < 1e-30f ? 0x1p100f : 1.f;
    const float width = hi * k - lo * k;
    const float sc = width > 0.f ? (float)LS_BINS / width : 0.f;
    auto bin_of = [&](float l) { return min(LS_BINS - 1, (int)((hi * k - l * k) * sc)); };
    for (int i = tid; i < LS_BINS; i += SMP_T) {
      sh.cnt[i] = 0;
      sh.wgt[i] = 0;
    }
    if (tid == 0) {
      sh.n = 0;
      sh.bin = LS_BINS;
    }
    __syncthreads();
    r.g.each([&](int, const Quad& q) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < q.n) {
          const float l = ls_clean(q.x[e]);
          if (l >= lo && l <= hi) {
            const int b = bin_of(l);
            atomicAdd(&sh.cnt[b], 1u);
            atomicAdd(&sh.wgt[b], r.fix(r.w(l)));
          }
        }
    });
    __syncthreads();
    // the first bin where the running count or mass reaches what is asked for
    static_assert(LS_BINS == 2 * SMP_T, "two bins a thread");
    const unsigned ca = sh.cnt[2 * tid], cb = sh.cnt[2 * tid + 1];
    const unsigned long long wa = sh.wgt[2 * tid], wb = sh.wgt[2 * tid + 1];
    unsigned long long ci = ls_scan((unsigned long long)(ca + cb), lane), wi = ls_scan(wa + wb, lane);
    if (lane == 63) {
      sh.cred[wave] = (unsigned)ci;
      sh.wred[wave] = wi;
    }
    __syncthreads();
    unsigned long long cbase = c0, wbase = w0;
    for (int x = 0; x < wave; ++x) {
      cbase += sh.cred[x];
      wbase += sh.wred[x];
    }
    ci += cbase;
    wi += wbase;
    auto reached = [&](unsigned long long c, unsigned long long w) { return by_weight ? (double)w >= need_w : c >= need_c; };
    if (reached(ci, wi)) {
      const int b = reached(ci - cb, wi - wb) ? 2 * tid : 2 * tid + 1;
      atomicMin(&sh.bin, b);
    }
    __syncthreads();
    const int bin = sh.bin;
    if (bin == LS_BINS) {  // everything is kept
      if (tid == SMP_T - 1) {
        sh.c0 = (unsigned)ci;
        sh.w0 = wi;
        sh.bv = floor_l;
        sh.bi = 0x7fffffff;
      }
      __syncthreads();
      return;
    }
    if (bin >> 1 == tid) {
      const bool odd = bin & 1;
      sh.c0 = (unsigned)(ci - cb - (odd ? 0 : ca));
      sh.w0 = wi - wb - (odd ? 0 : wa);
    }
    // the bin's codes: a list, and the range of their logits
    float mn = INFINITY, mx = -INFINITY;
    r.g.each([&](int v, const Quad& q) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < q.n) {
          const float l = ls_clean(q.x[e]);
          if (l >= lo && l <= hi && bin_of(l) == bin) {
            mn = fminf(mn, l);
            mx = fmaxf(mx, l);
            const int at = atomicAdd(&sh.n, 1);
            if (at < LS_LIST) {
              sh.lv[at] = l;
              sh.li[at] = v + e;
              sh.lw[at] = r.fix(r.w(l));
            }
          }
        }
    });
    for (int o = 32; o > 0; o >>= 1) {
      mn = fminf(mn, __shfl_xor(mn, o));
      mx = fmaxf(mx, __shfl_xor(mx, o));
    }
    if (lane == 0) {
      sh.fmn[wave] = mn;
      sh.fmx[wave] = mx;
    }
    __syncthreads();
    const int n = sh.n;
    c0 = sh.c0;
    w0 = sh.w0;
    for (int x = 0; x < SMP_W; ++x) {
      mn = fminf(mn, sh.fmn[x]);
      mx = fmaxf(mx, sh.fmx[x]);
    }
    if (n <= LS_LIST) {
      // rank the list: `parts` threads share a code's comparisons
      for (int i = tid; i < n; i += SMP_T) {
        sh.lc[i] = 0;
        sh.lb[i] = 0;
      }
      __syncthreads();
      int pad = 1;
      while (pad < n) pad <<= 1;
      const int parts = SMP_T / pad, i = tid & (pad - 1), part = tid / pad;
      if (i < n) {
        const float li = sh.lv[i];
        const int ii = sh.li[i];
        unsigned c = 0;
        unsigned long long w = 0;
        for (int j = part; j < n; j += parts)
          if (sh.lv[j] > li || (sh.lv[j] == li && sh.li[j] < ii)) {
            ++c;
            w += sh.lw[j];
          }
        atomicAdd(&sh.lc[i], c);
        atomicAdd(&sh.lb[i], w);
      }
      __syncthreads();
      // the one code with the bound inside it
      for (int k = tid; k < n; k += SMP_T) {
        const unsigned c = c0 + sh.lc[k];
        const unsigned long long w = w0 + sh.lb[k];
        if (!reached(c, w) && reached(c + 1, w + sh.lw[k])) {
          sh.bv = sh.lv[k];
          sh.bi = sh.li[k];
          sh.c0 = c + 1;
          sh.w0 = w + sh.lw[k];
        }
      }
      __syncthreads();
      return;
    }
    if (mn == mx) {
      // equal logits: so many of them, in code order
      const unsigned long long w1 = r.fix(r.w(mx));
      unsigned take;
      if (by_weight) {
        const double miss = need_w - (double)w0;
        take = w1 ? (unsigned)fmin(ceil(miss / (double)w1), (double)n) : (unsigned)n;
        take = max(take, 1u);
      } else {
        take = need_c - c0;
      }
      unsigned mine = 0;  // ties of this wave's segment, then those before it
      r.g.each([&](int, const Quad& q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) mine += __popcll(__ballot(e < q.n && ls_clean(q.x[e]) == mx));
      });
      if (lane == 0) sh.cred[wave] = mine;
      __syncthreads();
      unsigned at = 0;
      for (int x = 0; x < wave; ++x) at += sh.cred[x];
      r.g.each([&](int v, const Quad& q) {
        unsigned k = 0, all = 0;
        bool is[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          is[e] = e < q.n && ls_clean(q.x[e]) == mx;
          const uint64_t m = __ballot(is[e]);
          k += __popcll(m & ((1ull << lane) - 1));
          all += __popcll(m);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (is[e]) {
            if (at + k == take - 1) sh.bi = v + e;
            ++k;
          }
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
    hi = mx;
    lo = mn;
    __syncthreads();  // sh.n and sh.bin are read above and written at the top
  }
}

template <int NG>
__global__ __launch_bounds__(SMP_T) void sample_logits_kernel(SampleArgs a) {
  __shared__ LsShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x, V = a.V;
  const double T = a.temperatures ? (double)a.temperatures[row] : a.temperature;
  const int top_k = a.top_ks ? a.top_ks[row] : a.top_k;
  const double top_p = a.top_ps ? (double)a.top_ps[row] : a.top_p;
  const double min_any = a.min_ps ? (double)a.min_ps[row] : a.min_p;
  const double min_p = min_any > 1.0 ? 1.0 : min_any;  // the largest always stays (NaN: nothing is below it)
  const Seg<NG> g(a.logits + (size_t)row * a.ld, V);
  // largest logit, and the lowest code that has it
  float mx = -INFINITY;
  int am = 0x7fffffff;
  g.each([&](int v, const Quad& q) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < q.n) {
        const float l = ls_clean(q.x[e]);
        if (l > mx) {
          mx = l;
          am = v + e;
        }
      }
  });
  for (int o = 32; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(mx, o);
    const int a2 = __shfl_xor(am, o);
    if (m2 > mx || (m2 == mx && a2 < am)) {
      mx = m2;
      am = a2;
    }
  }
  if (lane == 0) {
    sh.fmx[wave] = mx;
    sh.ired[wave] = am;
  }
  __syncthreads();
  for (int x = 0; x < SMP_W; ++x)
    if (sh.fmx[x] > mx || (sh.fmx[x] == mx && sh.ired[x] < am)) {
      mx = sh.fmx[x];
      am = sh.ired[x];
    }
  __syncthreads();
  if (mx == -INFINITY || !(T > 0.0)) {  // nothing to draw, or the largest
    if (tid == 0) {
      a.tokens[row] = mx == -INFINITY ? -1 : am;
      if (a.probs) a.probs[row] = mx == -INFINITY ? 0.f : 1.f;
    }
    return;
  }
  const LsRow<NG> r(g, mx, fmin(1.0 / T, 1e300));
  // logits below this have no weight (45 and one binary places: 32 > 46 ln 2), and min_p's own bound lies above it or
  // is met by the weight itself
  const float floor_l = fmaxf((float)((double)mx - 32.0 * T), -3.4028234664e38f);
  float bv = floor_l;
  int bi = 0x7fffffff;
  double mass = -1.0;
  if (top_k > 0 && top_k < V) {
    ls_bound(r, floor_l, false, (unsigned)top_k, 0.0, sh);
    bv = sh.bv;
    bi = sh.bi;
    mass = (double)sh.w0;
    __syncthreads();
  }
  auto kept = [&](float l, int v) { return l > bv || (l == bv && v <= bi); };
  auto block_sum = [&](unsigned long long s) {  // inclusive over the waves before and this one, then all
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) sh.wred2[wave] = s;
    __syncthreads();
    unsigned long long t = 0;
    for (int x = 0; x < SMP_W; ++x) t += sh.wred2[x];
    return t;
  };
  if (top_p < 1.0) {
    if (mass < 0.0) {
      unsigned long long s = 0;
      g.each([&](int, const Quad& q) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < q.n) {
            const float l = ls_clean(q.x[e]);
            if (l >= floor_l) s += r.fix(r.w(l));
          }
      });
      mass = (double)block_sum(s);
      __syncthreads();
    }
    // the prefix of the first mass of top_p; with a top-k it ends inside that prefix
    const double need = fmax(top_p * mass, 1.0);
    ls_bound(r, floor_l, true, 0u, need, sh);
    bv = sh.bv;
    bi = sh.bi;
    __syncthreads();
  }
  // running sum over the kept codes in code order
  auto weight = [&](float l, int v) -> unsigned long long {
    if (!(l >= floor_l) || !kept(l, v)) return 0;
    const double w = r.w(l);
    return w < min_p ? 0 : r.fix(w);
  };
  unsigned long long s = 0;
  int last = -1;
  g.each([&](int v, const Quad& q) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < q.n) {
        const unsigned long long w = weight(ls_clean(q.x[e]), v + e);
        s += w;
        if (w) last = v + e;
      }
  });
  unsigned long long mine = s;
  for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
  const unsigned long long total = block_sum(s);
  unsigned long long base = 0;
  for (int x = 0; x < wave; ++x) base += sh.wred2[x];
  const double u = a.u[row];
  const double target = (u > 0.0 ? u : 0.0) * (double)total;
  for (int o = 32; o > 0; o >>= 1) last = max(last, __shfl_xor(last, o));
  if (lane == 0) sh.ired[wave] = last;
  if (tid == 0) sh.bi = 0x7fffffff;
  __syncthreads();
  // the wave whose running sum passes the target walks its codes
  if ((double)(base + mine) > target && !((double)base > target)) {
    unsigned long long run = base;
    bool found = false;
    int cand = 0x7fffffff;
    float cl = 0.f;
    g.each([&](int v, const Quad& q) {
      if (found) return;
      unsigned long long w[4], t = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = e < q.n ? weight(ls_clean(q.x[e]), v + e) : 0;
        t += w[e];
      }
      const unsigned long long inc = ls_scan(t, lane);
      unsigned long long c = run + (inc - t);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c += w[e];
        if (cand == 0x7fffffff && w[e] && (double)c > target) {
          cand = v + e;
          cl = ls_clean(q.x[e]);
        }
      }
      run += __shfl(inc, 63);
      found = __ballot(cand != 0x7fffffff) != 0;
    });
    int best = cand;
    for (int o = 32; o > 0; o >>= 1) best = min(best, __shfl_xor(best, o));
    if (cand == best && best != 0x7fffffff) {
      a.tokens[row] = cand;
      if (a.probs) a.probs[row] = (float)(r.w(cl) * LS_ONE / (double)total);
      sh.bi = cand;
    }
  }
  __syncthreads();
  if (sh.bi == 0x7fffffff && tid == 0) {  // u at or past one: the last kept code
    for (int x = 0; x < SMP_W; ++x) last = max(last, sh.ired[x]);
    a.tokens[row] = last;
    if (a.probs) a.probs[row] = (float)(r.w(ls_clean(a.logits[(size_t)row * a.ld + last])) * LS_ONE / (double)total);
  }
}

void sample_logits(const SampleArgs& a, hipStream_t st) {
  if (a.V <= 4 * SMP_HELD)
    hipLaunchKernelGGL(sample_logits_kernel<4>, dim3(a.R), dim3(SMP_T), 0, st, a);
  else if (a.V <= 8 * SMP_HELD)
    hipLaunchKernelGGL(sample_logits_kernel<8>, dim3(a.R), dim3(SMP_T), 0, st, a);
  else
    hipLaunchKernelGGL(sample_logits_kernel<0>, dim3(a.R), dim3(SMP_T), 0, st, a);
}

}  // namespace ssd
