// Drawing one token per row of logits with temperature, top-k, top-p and min-p from given uniforms.
//   Tokens in order: larger logit first, the lower index first among equals.  Kept are, of w_i = exp((z_i - max z) / T):
//     the first k (top_k > 0);  of those the shortest run from the first on whose sum of w reaches top_p times the sum of all of them (top_p < 1);
//     of those the ones with w_i >= min_p.  All three are runs from the first token on, so that "kept" is one comparison with a last (logit, index).
//   token = argmax over kept of z_i / T - log(-log u_i), the lowest index first: with u uniform, a draw with probabilities proportional to w_i.
//     (In log2 throughout: a factor and a constant that all scores share change nothing.)
//   T <= 0: the largest logit.  logprob = z_token - log sum_i exp z_i over all tokens, at temperature 1.
//   A logit of -inf or NaN is never drawn, +inf counts as the largest float; without a token that can be drawn: -1 and -inf.
// A row is one workgroup's, its first 128 KB wait in LDS between the passes.  A histogram over the range of logits in question finds where the
// count or the sum of w is reached: 2048 bins hold a count and the sum of w over the bin's largest possible w, in fixed point (2^-26), so that no
// order of additions matters.  Usually few tokens stand before the end of that bin: they go to a list, which is sorted, and what is left of
// the three rules and the draw look at nothing else.  Otherwise the bin is the next round's range, until its tokens fit a list of 256 that is ranked
// directly (equal logits are told apart by histograms over their indices), and the draw goes over the row once more.
#include <float.h>

#include "kernels.h"
#include "wave_math.h"

namespace hydra {
namespace {

constexpr int NT = 1024, NB = 2048, CAP = 256, LIST = 2048;
constexpr int ROW_BYTES = 131072;  // of a row in LDS
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -__builtin_inff();
constexpr float DEPTH = 24.f * LOG2E;  // the first round's bins reach down to w = e^-24; what is below goes to the last one
typedef unsigned long long u64;

struct Last { float z; int i; };  // the last kept token: kept are larger logits, and equal ones up to its index
__device__ __forceinline__ bool kept(const Last& t, float z, int i) { return z > t.z || (z == t.z && i <= t.i); }

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float logit(float z) { return z == z ? fminf(z, FLT_MAX) : NEG_INF; }

// an order of logits and indices as one of whole numbers: larger first
__device__ __forceinline__ u64 order_key(float z, int i) {
  const unsigned b = __float_as_uint(z + 0.f);  // -0 is 0
  return (u64)(b ^ ((int)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - (unsigned)i);
}
__device__ __forceinline__ float key_logit(u64 k) {
  const unsigned b = (unsigned)(k >> 32);
  return __uint_as_float(b ^ ((int)b < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_index(u64 k) { return (int)(0xffffffffu - (unsigned)k); }

struct Shared {
  union {
    u64 bin[NB];      // count << 45 | sum of w / (largest w of the bin), 2^-26
    u64 list[LIST];   // order keys
    struct { u64 key[CAP], w[CAP]; } some;
  };
  float part_a[NT / 64];
  int part_i[NT / 64];
  unsigned part_n[NT / 64];
  u64 part_w[NT / 64];
  int n, at, found_i;
  unsigned above_n, here_n;
  u64 above_w, run_w;
  float found_z;
  float best_z;
};

// The row's tokens, 16 bytes at a time: those in LDS, then those that are read again.
template <typename T>
struct Row {
  static constexpr int VEC = 16 / sizeof(T);
  const T* p;
  uint4* lds;
  int V, n_vec, n_lds;  // tokens; runs of VEC of them, the last one perhaps in part; runs in LDS
  bool wide, odd;       // 16-byte loads; some logit is NaN or +inf
  __device__ __forceinline__ uint4 load(int q) const {
    if (wide && (q + 1) * VEC <= V) return *reinterpret_cast<const uint4*>(p + (size_t)q * VEC);
    uint32_t w[4];
    if constexpr (VEC == 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = q * 4 + e < V ? __float_as_uint(p[q * 4 + e]) : 0xff800000u;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = (q * 8 + 2 * e < V ? (uint32_t)p[q * 8 + 2 * e] : 0xff80u) | (q * 8 + 2 * e + 1 < V ? (uint32_t)p[q * 8 + 2 * e + 1] : 0xff80u) << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  template <bool FIX, typename F>
  static __device__ __forceinline__ void tokens(const uint4& v, int q, F& f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (VEC == 4) {
        const float z = __uint_as_float(w[e]);
        f(FIX ? logit(z) : z, q * 4 + e);
      } else {
        const float a = __uint_as_float(w[e] << 16), b = __uint_as_float(w[e] & 0xffff0000u);
        f(FIX ? logit(a) : a, q * 8 + 2 * e);
        f(FIX ? logit(b) : b, q * 8 + 2 * e + 1);
      }
    }
  }
  // Every token once: f(logit, index).  Tokens past the row's end are -inf.  Four loads from memory are under way together.
  template <bool FIX, typename F>
  __device__ __forceinline__ void all(F& f) const {
    for (int q = threadIdx.x; q < n_lds; q += NT) tokens<FIX>(lds[q], q, f);
    for (int q0 = n_lds + threadIdx.x; q0 < n_vec; q0 += 4 * NT) {
      uint4 v[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) v[s] = q0 + s * NT < n_vec ? load(q0 + s * NT) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (q0 + s * NT < n_vec) tokens<FIX>(v[s], q0 + s * NT, f);
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if (odd) all<true>(f);
    else all<false>(f);
  }
  // The first pass: what LDS holds goes there; f as in all(), with the logits as they are.
  template <typename F>
  __device__ __forceinline__ void first(F f) const {
    for (int q0 = threadIdx.x; q0 < n_vec; q0 += 8 * NT) {
      uint4 v[8];
#pragma unroll
      for (int s = 0; s < 8; ++s) v[s] = q0 + s * NT < n_vec ? load(q0 + s * NT) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const int q = q0 + s * NT;
        if (q < n_lds) lds[q] = v[s];
        if (q < n_vec) tokens<false>(v[s], q, f);
      }
    }
  }
};

__device__ __forceinline__ float block_max(float v, float* part) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return wave_max(part[threadIdx.x & (NT / 64 - 1)]);
}
__device__ __forceinline__ float block_sum(float v, float* part) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = part[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) r += part[i];
  return r;
}
__device__ __forceinline__ u64 fixed(float w) { return (u64)(w * 17592186044416.f); }  // 2^44

// Sums of everything up to and with this thread's (n, w), in thread order; total: over all threads.
__device__ __forceinline__ void block_scan(unsigned& n, u64& w, unsigned& total_n, u64& total_w, Shared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned pn = __shfl_up(n, d);
    const u64 pw = __shfl_up(w, d);
    if (lane >= d) n += pn, w += pw;
  }
  __syncthreads();
  if (lane == 63) sh.part_n[wave] = n, sh.part_w[wave] = w;
  __syncthreads();
  total_n = 0, total_w = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i == wave) n += total_n, w += total_w;
    total_n += sh.part_n[i], total_w += sh.part_w[i];
  }
}

// One round's histogram and where its sums reach what is asked.
struct Range {
  float hi, lo, low;   // logits in it: lo .. hi; the bins end at low
  bool ties;           // all that is in it has the logit hi: bins of indices
  int i_lo, i_n;
  float c;             // bins per unit
  unsigned per;        // indices per bin
  __device__ __forceinline__ void begin() {
    c = fminf(fmaxf((float)NB / (hi - low), 1e-37f), FLT_MAX);
    per = (unsigned)(i_n + NB - 1) / NB;
  }
  __device__ __forceinline__ bool in(const Last& t, float z, int i) const {
    return z <= hi && z >= lo && kept(t, z, i) && (!ties || (i >= i_lo && i < i_lo + i_n));
  }
  // the largest logit is alone in the first bin, so that every round takes something out of the next one's range
  __device__ __forceinline__ int bin_of(float z, int i) const {
    return ties ? (int)((unsigned)(i - i_lo) / per) : z == hi ? 0 : (int)fminf(fmaxf((hi - z) * c, 1.f), (float)(NB - 1));
  }
};
__device__ __forceinline__ void clear(Shared& sh) {
  __syncthreads();
  for (int i = threadIdx.x; i < NB; i += NT) sh.bin[i] = 0;
  if (threadIdx.x == 0) sh.n = 0, sh.at = -1;
  __syncthreads();
}
// inv: log2(e) / T; a bin's largest weight is that of its upper edge
__device__ __forceinline__ float edge(const Range& g, int bin, float zmax, float inv) { return (g.hi - zmax) * inv - (g.ties || !bin ? 0.f : (float)bin * (inv / g.c)); }
__device__ __forceinline__ u64 entry(const Range& g, int bin, float z, float zmax, float inv, bool mass) {
  constexpr u64 ONE = 1ull << 45;
  if (!mass) return ONE;
  return ONE + (u64)(unsigned)(fminf(exp2_hw((z - zmax) * inv - edge(g, bin, zmax, inv)), 2.f) * 67108864.f);
}
// sh.at: the first bin through which the sum of counts (by_mass: of weights) reaches k (p times `of`, or times the sum of all bins where `of` is 0);
// -1 where none does.  sh.above_*: the sums before it; sh.here_n: its count; returns the target that the sum of weights was held against.
__device__ __forceinline__ u64 find_bin(const Range& g, Shared& sh, float zmax, float inv, bool mass, bool by_mass, unsigned k, u64 target, float p) {
  const int b = 2 * (int)threadIdx.x;
  __syncthreads();
  const u64 e0 = sh.bin[b], e1 = sh.bin[b + 1];
  const unsigned n0 = (unsigned)(e0 >> 45), n1 = (unsigned)(e1 >> 45);
  u64 w0 = 0, w1 = 0;
  if (mass) {
    constexpr double UNIT = 262144.;  // 2^44 / 2^26
    constexpr u64 LOW = (1ull << 45) - 1;
    w0 = (u64)((double)(e0 & LOW) * ((double)exp2_hw(edge(g, b, zmax, inv)) * UNIT));
    w1 = (u64)((double)(e1 & LOW) * ((double)exp2_hw(edge(g, b + 1, zmax, inv)) * UNIT));
  }
  unsigned n = n0 + n1, all_n;
  u64 w = w0 + w1, all_w;
  const unsigned an = sh.above_n;
  const u64 aw = sh.above_w;
  block_scan(n, w, all_n, all_w, sh);
  if (p >= 0.f) {
    const double want = __builtin_ceil((double)p * (double)all_w);
    target = want < 1.0 ? 1ull : (u64)want;
  }
  n += an, w += aw;
  // sums through the end of bin b, and through b + 1
  const unsigned na = n - n1;
  const u64 wa = w - w1;
  const bool here0 = by_mass ? wa - w0 < target && wa >= target : na - n0 < k && na >= k;
  const bool here1 = by_mass ? wa < target && w >= target : na < k && n >= k;
  if (here0) sh.at = b, sh.above_n = na - n0, sh.above_w = wa - w0, sh.here_n = n0;
  if (here1) sh.at = b + 1, sh.above_n = na, sh.above_w = wa, sh.here_n = n1;
  __syncthreads();
  return target;
}

// The last token of the run that reaches k tokens, or the mass `target`, among those kept by `t`; t itself where nothing does.  begun: the first
// round's histogram stands in sh and find_bin has been called.  sh.run_w: the run's mass, where it is found (sh.found_i >= 0).
template <typename R>
__device__ __forceinline__ Last find_last(const R& row, Shared& sh, Range g, bool begun, Last t, float zmax, float inv, bool by_mass, unsigned k, u64 target,
                                          bool mass) {
  const int tid = threadIdx.x;
  while (true) {
    if (!begun) {
      g.begin();
      clear(sh);
      row.each([&](float z, int i) {
        if (g.in(t, z, i)) {
          const int bin = g.bin_of(z, i);
          atomicAdd(&sh.bin[bin], entry(g, bin, z, zmax, inv, mass));
        }
      });
      find_bin(g, sh, zmax, inv, mass, by_mass, k, target, -1.f);
    }
    begun = false;
    const int bin = sh.at;
    if (tid == 0) sh.found_i = -1, sh.n = 0;
    __syncthreads();
    if (bin < 0) return t;
    const unsigned n = sh.here_n;
    if (n <= CAP) {
      row.each([&](float z, int i) {
        if (g.in(t, z, i) && g.bin_of(z, i) == bin) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < CAP) sh.some.key[at] = order_key(z, i), sh.some.w[at] = mass ? fixed(exp2_hw((z - zmax) * inv)) : 0;
        }
      });
      __syncthreads();
      if (tid < (int)n) {
        const u64 key = sh.some.key[tid], own = sh.some.w[tid];
        unsigned before = sh.above_n;
        u64 w = sh.above_w;
        for (unsigned q = 0; q < n; ++q)
          if (sh.some.key[q] > key) ++before, w += sh.some.w[q];
        if (by_mass ? w < target && w + own >= target : before == k - 1) sh.found_z = key_logit(key), sh.found_i = key_index(key), sh.run_w = w + own;
      }
      __syncthreads();
      return sh.found_i < 0 ? t : Last{sh.found_z, sh.found_i};
    }
    if (g.ties) {
      g.i_lo += bin * g.per, g.i_n = min((int)g.per, g.i_n - bin * (int)g.per);
      continue;
    }
    float most = NEG_INF, least = NEG_INF;  // the range of what is in the bin (the smaller one with its sign turned)
    row.each([&](float z, int i) {
      if (g.in(t, z, i) && g.bin_of(z, i) == bin) most = fmaxf(most, z), least = fmaxf(least, -z);
    });
    g.hi = block_max(most, sh.part_a);
    g.lo = g.low = -block_max(least, sh.part_a);
    g.ties = g.hi == g.lo;
  }
}

// Larger keys first.  n keys, room for the next power of two.
__device__ __forceinline__ void sort_keys(u64* key, int n) {
  int m = 64;
  while (m < n) m <<= 1;
  for (int i = n + (int)threadIdx.x; i < m; i += NT) key[i] = 0;
  for (int k = 2; k <= m; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      __syncthreads();
      for (int p = threadIdx.x; p < m / 2; p += NT) {
        const int a = (p & ~(j - 1)) * 2 | (p & (j - 1)), b = a | j;  // the pair whose numbers differ in j
        const u64 x = key[a], y = key[b];
        if ((x < y) == !(a & k)) key[a] = y, key[b] = x;
      }
    }
  __syncthreads();
}

struct Best { float s, z; int i; };
__device__ __forceinline__ void race(Best& b, float z, int i, float zmax, float inv, const float* u) {
  const float s = fmaxf((z - zmax) * inv - __builtin_amdgcn_logf(-__builtin_amdgcn_logf(fminf(u[i], 0.99999994f))), -FLT_MAX);
  if (s > b.s || (s == b.s && i < b.i)) b = {s, z, i};
}

template <typename T>
__global__ __launch_bounds__(NT) void sample_kernel(const SampleArgs a) {
  __shared__ Shared sh;
  extern __shared__ __attribute__((aligned(16))) uint4 row_lds[];
  const int g = blockIdx.y, r = blockIdx.x, tid = threadIdx.x;
  Row<T> row;
  row.V = a.V;
  row.p = static_cast<const T*>(a.z[g]) + (size_t)r * a.ldz;
  row.lds = row_lds;
  row.n_vec = (a.V + Row<T>::VEC - 1) / Row<T>::VEC;
  row.n_lds = min(row.n_vec, ROW_BYTES / 16);
  row.wide = (uintptr_t)row.p % 16 == 0;
  const float temp = a.temperature[r], top_p = a.top_p[r], min_p = fminf(a.min_p[r], 1.f);
  const int top_k = a.top_k[r];
  const bool greedy = !(temp > 0.f);
  float most = NEG_INF;
  bool odd = false;
  row.first([&](float z, int) {
    most = fmaxf(most, z);
    odd |= !(z <= FLT_MAX);
  });
  if (tid == 0) sh.n = 0, sh.above_n = 0, sh.above_w = 0;
  const float zmax = fminf(block_max(most, sh.part_a), FLT_MAX);
  if (odd) sh.n = 1;
  __syncthreads();
  row.odd = sh.n;
  if (zmax == NEG_INF) {
    if (tid == 0) {
      a.token[g][r] = -1;
      if (a.logprob[g]) a.logprob[g][r] = NEG_INF;
    }
    return;
  }
  const float by = greedy ? 1.f : fminf(fmaxf(1.0f / temp, 1e-30f), 1e30f), inv = LOG2E * by;
  const float* u = a.u[g] + (size_t)r * a.ldu;
  const bool by_k = !greedy && top_k > 0 && top_k < a.V, by_p = !greedy && top_p < 1.f;
  const bool want_lse = a.logprob[g] != nullptr;
  float lse = 0.f;
  Best best = {NEG_INF, NEG_INF, 0x7fffffff};
  if (!by_k && !by_p) {  // one pass
    row.each([&](float z, int i) {
      if (want_lse) lse += exp2_hw((z - zmax) * LOG2E);
      if (greedy ? z == zmax && i < best.i : z > NEG_INF && (min_p <= 0.f || exp2_hw((z - zmax) * inv) >= min_p)) {
        if (greedy) best = {0.f, z, i};
        else race(best, z, i, zmax, inv, u);
      }
    });
  } else {
    Range range = {zmax, -FLT_MAX, fmaxf(zmax - DEPTH / inv, -FLT_MAX), false, 0, a.V, 0.f, 0};
    range.begin();
    clear(sh);
    row.each([&](float z, int i) {
      if (want_lse) lse += exp2_hw((z - zmax) * LOG2E);
      if (z > NEG_INF) {
        const int bin = range.bin_of(z, i);
        atomicAdd(&sh.bin[bin], entry(range, bin, z, zmax, inv, by_p));
      }
    });
    // both rules end at or before where the first one does: the k-th token, or without top-k the share of all mass
    u64 target = find_bin(range, sh, zmax, inv, by_p, !by_k, (unsigned)top_k, 0, by_k ? -1.f : fmaxf(top_p, 0.f));
    const unsigned n = sh.at >= 0 ? sh.above_n + sh.here_n : LIST + 1;
    if (n <= LIST) {
      const int bin = sh.at;
      __syncthreads();
      row.each([&](float z, int i) {
        if (z > NEG_INF && range.bin_of(z, i) <= bin) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < LIST) sh.list[at] = order_key(z, i);
        }
      });
      sort_keys(sh.list, (int)n);
      unsigned none = 0, x_n;
      u64 w[2], run = 0, all;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = 2 * tid + e;
        w[e] = at < (int)n && (!by_k || at < top_k) ? fixed(exp2_hw((key_logit(sh.list[at]) - zmax) * inv)) : 0;
        run += w[e];
      }
      if (by_p) {
        block_scan(none, run, x_n, all, sh);
        if (by_k) {
          const double want = __builtin_ceil((double)fmaxf(top_p, 0.f) * (double)all);
          target = want < 1.0 ? 1ull : (u64)want;
        }
        run -= w[0] + w[1];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = 2 * tid + e;
        if (at < (int)n && (!by_k || at < top_k) && (!by_p || run < target)) {
          const float z = key_logit(sh.list[at]);
          if (exp2_hw((z - zmax) * inv) >= min_p) race(best, z, key_index(sh.list[at]), zmax, inv, u);
        }
        run += w[e];
      }
    } else {
      Last t = {-FLT_MAX, 0x7fffffff};
      t = find_last(row, sh, range, true, t, zmax, inv, !by_k, (unsigned)top_k, target, by_p);
      if (by_k && by_p) {
        u64 total = sh.run_w;
        if (sh.found_i < 0) {  // fewer than k tokens can be drawn: all of them are kept
          u64 w = 0, x_w;
          unsigned x = 0, x_n;
          row.each([&](float z, int) { w += fixed(exp2_hw((z - zmax) * inv)); });
          block_scan(x, w, x_n, x_w, sh);
          total = x_w;
        }
        const double want = __builtin_ceil((double)fmaxf(top_p, 0.f) * (double)total);
        __syncthreads();
        if (tid == 0) sh.above_n = 0, sh.above_w = 0;
        t = find_last(row, sh, range, false, t, zmax, inv, true, 0, want < 1.0 ? 1ull : (u64)want, true);
      }
      row.each([&](float z, int i) {
        if (z > NEG_INF && kept(t, z, i) && exp2_hw((z - zmax) * inv) >= min_p) race(best, z, i, zmax, inv, u);
      });
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const Best o = {__shfl_xor(best.s, d), __shfl_xor(best.z, d), __shfl_xor(best.i, d)};
    if (o.s > best.s || (o.s == best.s && o.i < best.i)) best = o;
  }
  if (want_lse) lse = block_sum(lse, sh.part_a);
  __syncthreads();
  if ((tid & 63) == 0) sh.part_a[tid >> 6] = best.s, sh.part_i[tid >> 6] = best.i, sh.part_n[tid >> 6] = __float_as_uint(best.z);
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < NT / 64; ++i)
      if (sh.part_a[i] > best.s || (sh.part_a[i] == best.s && sh.part_i[i] < best.i)) best = {sh.part_a[i], __uint_as_float(sh.part_n[i]), sh.part_i[i]};
    a.token[g][r] = best.i;
    if (want_lse) a.logprob[g][r] = best.z - zmax - __builtin_amdgcn_logf(lse) * LN2;
  }
}

}  // namespace

const char* sample_refusal(const SampleArgs& a) {
  if (a.rows < 1 || a.V < 1) return "rows and V are at least 1";
  if (a.V > (1 << 18)) return "V is 262144 at most";
  if (a.ldz < a.V || a.ldu < a.V) return "ldz or ldu is less than V";
  return nullptr;
}

hipError_t sample_init() {
  hipError_t e = hipFuncSetAttribute((const void*)sample_kernel<float>, hipFuncAttributeMaxDynamicSharedMemorySize, ROW_BYTES);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)sample_kernel<bf16_t>, hipFuncAttributeMaxDynamicSharedMemorySize, ROW_BYTES);
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  const size_t esize = a.dtype == GEMM_F32 ? 4 : 2, row = ((size_t)a.V * esize + 15) / 16 * 16;
  const unsigned lds = (unsigned)(row < ROW_BYTES ? row : ROW_BYTES);
  const dim3 grid(a.rows, a.G);
  if (a.dtype == GEMM_F32) hipLaunchKernelGGL((sample_kernel<float>), grid, dim3(NT), lds, s, a);
  else hipLaunchKernelGGL((sample_kernel<bf16_t>), grid, dim3(NT), lds, s, a);
  return hipGetLastError();
}

}  // namespace hydra
