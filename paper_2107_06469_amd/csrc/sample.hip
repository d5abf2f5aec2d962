// Drawing one token per row of logits with temperature, top-k, top-p and min-p from given uniforms.
//   Tokens in order: larger logit first, the lower index first among equals.  Kept are, of w_i = exp((z_i - max z) / T):
//     the first k (top_k > 0);  of those the shortest run from the first on whose sum of w reaches top_p times the sum of all of them (top_p < 1);
//     of those the ones with w_i >= min_p.  All three are runs from the first token on, so that "kept" is one comparison with a last (logit, index).
//   token = argmax over kept of z_i / T - log(-log u_i), the lowest index first: with u uniform, a draw with probabilities proportional to w_i.
//     (In log2 throughout: a factor and a constant that all scores share change nothing.)
//   T <= 0: the largest logit.  logprob = z_token - log sum_i exp z_i over all tokens, at temperature 1.
//   A logit of -inf or NaN is never drawn, +inf counts as the largest number of the logits' type; without a token that can be drawn: -1 and -inf.
// A row is one workgroup's; it waits in LDS between the passes, or as much of it as fits.  A histogram over the range of logits finds where the count or
// the sum of w is reached: 2048 bins hold a count and the sum of w over the bin's largest possible w, in fixed point (2^-26), so that no order of
// additions matters.  Usually at most 4096 tokens (8192 of a row that LDS does not hold) stand before the end of that bin: their indices go to a
// list, and what is left of the rules and the draw look at nothing else.  Up to 128 of them are ranked directly; of more, or over the whole row, the
// bin is the next round's range until 256 tokens at most are left in it (equal logits are told apart by histograms over their indices).
// Where the list's tokens are known without the histogram it is left out: those that min_p leaves, and for a small top_k those at or above the top_k-th of
// the threads' largest logits.
// Bound by one CU's vector unit, each instruction a token being 2048 cycles of 131072 tokens, and LDS atomics, for many rows: 256 of 131072 in bf16
// with top-p and min-p 35 us, 1.9 TB/s (50 to 60 where the smallest min-p leaves more than the list holds); 2 x 64 of 32000 in fp32 with mixed rules 35,
// of which a row with a top-k of 1500 and top-p takes 27.  A single row of 32000 with a top-k of 50 and top-p takes 13, a chain of passes and barriers.  With the histogram for these too, the 256 rows take 142 and the single
// one 17.  Rows that do not fit LDS are read again, through the caches.  A kept set larger than the list costs another pass, over the uniforms
// too (131072 tokens, top-p 0.97 alone: 115 us).
#include <float.h>

#include "kernels.h"
#include "wave_math.h"

namespace hydra {
namespace {

constexpr int NT = 1024, NB = 2048, CAP = 256, FEW = 128;
// Up to this top_k it cuts first: the list is then short enough to be ranked directly, mostly (larger ones take longer that way: 1500 with top-p 30 us
// instead of 26).  Bins of the threads' largest logits that tell where.
constexpr int SMALL_K = 96, NC = 256;
// A row's bytes and the listed tokens share LDS: a row that fits leaves room for 4096 tokens, of one that does not less waits there for 8192 (256 rows of 131072 in
// bf16 at temperature 1.3, a min-p of 0.0008: 49 us, with 4096 and more of the row 92).
constexpr int ROW_BYTES = 129024, LIST = 4096, WIDE_ROW_BYTES = ROW_BYTES - 4 * LIST, WIDE_LIST = 2 * LIST;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -__builtin_inff();
constexpr float DEPTH = 24.f * LOG2E;  // the first round's bins reach down to w = e^-24; what is below goes to the last one
typedef unsigned long long u64;

struct Last { float z; int i; };  // the last kept token: kept are larger logits, and equal ones up to its index
__device__ __forceinline__ bool kept(const Last& t, float z, int i) { return z > t.z || (z == t.z && i <= t.i); }

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

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
  u64 bin[NB];      // count << 45 | sum of w / (largest w of the bin), 2^-26
  unsigned top[NC];  // threads by their largest logit
  float part_a[NT / 64], part_b[NT / 64], part_z[NT / 64];
  int part_i[NT / 64];
  unsigned part_n[NT / 64];
  double part_w[NT / 64];
  int n, runs, at, odd, found_i;
  unsigned above_n, here_n;
  double above_w, run_w;
  float found_z;
};
// up to CAP tokens that are ranked, in the bins' place
struct Some { u64 key[CAP], w[CAP]; };
static_assert(sizeof(Some) <= NB * sizeof(u64), "the ranked tokens take the bins' place");

// The row's tokens, 16 bytes at a time: those in LDS, then those that are read again.
template <typename T>
struct Row {
  static constexpr int VEC = 16 / sizeof(T);
  // What +inf counts as wherever a logit is looked at: the largest number of the type, so that a run of 16 bytes can hold it.
  static constexpr float TOP = VEC == 4 ? FLT_MAX : 0x1.fep127f;
  static __device__ __forceinline__ float logit(float z) { return z == z ? fminf(z, TOP) : NEG_INF; }
  const T* p;
  uint4* lds;
  int V, n_vec, n_lds;  // tokens; runs of VEC of them, the last one perhaps in part; runs in LDS
  bool wide, odd;       // 16-byte loads; some logit, or the rest of the last run, is no finite number
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
  __device__ __forceinline__ float at(int i) const {
    if constexpr (VEC == 4) return logit(i < n_lds * VEC ? reinterpret_cast<const float*>(lds)[i] : p[i]);
    else return logit(__uint_as_float((uint32_t)(i < n_lds * VEC ? reinterpret_cast<const bf16_t*>(lds)[i] : p[i]) << 16));
  }
  // NaN to -inf and +inf to TOP, in a run
  static __device__ __forceinline__ uint4 mended(uint4 v) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (VEC == 4) {
        w[e] = __float_as_uint(logit(__uint_as_float(w[e])));
      } else {
        const uint32_t lo = __float_as_uint(logit(__uint_as_float(w[e] << 16))), hi = __float_as_uint(logit(__uint_as_float(w[e] & 0xffff0000u)));
        w[e] = lo >> 16 | (hi & 0xffff0000u);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ uint4 run(int q) const { return q < n_lds ? lds[q] : load(q); }
  // f(logit, number in the run)
  template <typename F>
  static __device__ __forceinline__ void tokens(const uint4& v, F&& f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (VEC == 4) {
        f(__uint_as_float(w[e]), e);
      } else {
        f(__uint_as_float(w[e] << 16), 2 * e);
        f(__uint_as_float(w[e] & 0xffff0000u), 2 * e + 1);
      }
    }
  }
  // Every run once: f(run, number); tokens past the row's end are -inf.  The next run is asked for before this one's work, which stands here
  // once: a pass of several copies of it does not fit the instruction cache.
  template <typename F>
  __device__ __forceinline__ void runs(F f) const {
    int q = threadIdx.x;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (q < n_vec) v = run(q);
#pragma unroll 1
    while (q < n_vec) {
      const int at = q;
      uint4 now = v;
      q += NT;
      if (q < n_vec) v = run(q);
      if (odd) now = mended(now);
      f(now, at);
    }
  }
  // The same by tokens: f(logit, index).
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    runs([&](const uint4& v, int q) { tokens(v, [&](float z, int e) { f(z, q * VEC + e); }); });
  }
  // The first pass: what LDS holds goes there; f(logit, number in the run), with the logits as they are.
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
        if (q < n_vec) tokens(v[s], f);
      }
    }
  }
};

// All tokens of a row, or the listed ones.
template <typename T>
struct Tokens {
  const Row<T>& row;
  const unsigned* list;
  int n;
  bool listed;
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if (!listed) {
      row.each(f);
    } else {
#pragma unroll 1
      for (int e = threadIdx.x; e < n; e += NT) f(row.at((int)list[e]), (int)list[e]);
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
// Sums of weights do not depend on their order: a token's weight is a whole number of 2^-44, a bin's one of 2^-34 (of which a double holds 2^19
// exactly, and all tokens together weigh 2^18 at most).
__device__ __forceinline__ u64 fixed(float w) { return (u64)(w * 17592186044416.f); }
__device__ __forceinline__ double bin_units(u64 w) { return (double)w * (1.0 / 1024.0); }
constexpr double BIN_ONE = 17179869184.0;

// In the order of the first NS threads (whole waves; the others only come along): the sums of (n, w) before this thread's, and the sum of all w.
// A step that every wave takes costs a SIMD four times what it costs one wave: bookkeeping is left to four of them.
constexpr int NS = 256;
__device__ __forceinline__ void block_scan(unsigned n, double w, unsigned& before_n, double& before_w, double& all_w, Shared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  before_n = 0, before_w = 0;
  if (threadIdx.x < NS) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned pn = __shfl_up(n, d);
      const double pw = __shfl_up(w, d);
      if (lane >= d) n += pn, w += pw;
    }
    if (lane == 63) sh.part_n[wave] = n, sh.part_w[wave] = w;
    before_n = __shfl_up(n, 1), before_w = __shfl_up(w, 1);
    if (!lane) before_n = 0, before_w = 0;
  }
  __syncthreads();
  all_w = 0;
#pragma unroll
  for (int i = 0; i < NS / 64; ++i) {
    if (i < wave) before_n += sh.part_n[i], before_w += sh.part_w[i];
    all_w += sh.part_w[i];
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
  // after the first round the largest logit is alone in the first bin, so that every round takes something out of the next one's range
  bool first;
  __device__ __forceinline__ int bin_of(float z, int i) const {
    return ties ? (int)((unsigned)(i - i_lo) / per) : (int)fminf(fmaxf((hi - z) * c, first || z == hi ? 0.f : 1.f), (float)(NB - 1));
  }
};
__device__ __forceinline__ void clear(Shared& sh) {
  for (int i = threadIdx.x; i < NB / 2; i += NT) reinterpret_cast<uint4*>(sh.bin)[i] = make_uint4(0, 0, 0, 0);
  if (threadIdx.x == 0) sh.at = -1;
}
// inv: log2(e) / T; a bin's largest weight is that of its upper edge
__device__ __forceinline__ float edge(const Range& g, int bin, float zmax, float inv) { return (g.hi - zmax) * inv - (g.ties || !bin ? 0.f : (float)bin * (inv / g.c)); }
// sh.at: the first bin through which the sum of counts (by_mass: of weights) reaches k (the target; with p >= 0 that is p times the sum of all bins);
// it stays -1 where none does.  sh.above_*: the sums before it; sh.here_n: its count; returns the target.
__device__ __forceinline__ double find_bin(const Range& g, Shared& sh, float zmax, float inv, bool mass, bool by_mass, unsigned k, double target, float p, double& total) {
  constexpr int PER = NB / NS;
  const bool one = threadIdx.x < NS;
  const int b = one ? PER * (int)threadIdx.x : 0;
  __syncthreads();
  unsigned n[PER], all_n = 0;
  double w[PER], all_w = 0;
  if (one) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const u64 e = sh.bin[b + i];
      n[i] = (unsigned)(e >> 45);
      w[i] = 0;
      if (mass && n[i])  // two conversions: the sum has 45 bits
        w[i] = rint(((double)((unsigned)(e >> 32) & 0x1fffu) * 4294967296.0 + (double)(unsigned)e) *
                    ((double)exp2_hw(edge(g, b + i, zmax, inv)) * (BIN_ONE / 67108864.0)));
      all_n += n[i], all_w += w[i];
    }
  }
  unsigned cn;
  double cw;
  const unsigned an = sh.above_n;
  const double aw = sh.above_w;
  block_scan(all_n, all_w, cn, cw, total, sh);
  if (p >= 0.f) target = (double)p * total;
  cn += an, cw += aw;
  if (one) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned nn = cn + n[i];
      const double nw = cw + w[i];
      if (by_mass ? cw < target && nw >= target : cn < k && nn >= k) sh.at = b + i, sh.above_n = cn, sh.above_w = cw, sh.here_n = n[i];
      cn = nn, cw = nw;
    }
  }
  __syncthreads();
  return target;
}

// The last token of the run that reaches k tokens, or the mass `target`, among those kept by `t`; t itself where nothing does.  begun: the first
// round's histogram has been taken and find_bin called.  sh.run_w: the run's mass, where it is found (sh.found_i >= 0).
template <typename R>
__device__ __forceinline__ Last find_last(const R& row, Shared& sh, Range g, bool begun, Last t, float zmax, float inv, bool by_mass, unsigned k, double target,
                                          bool mass) {
  const int tid = threadIdx.x;
  Some& some = *reinterpret_cast<Some*>(sh.bin);
  while (true) {
    if (!begun) {
      g.begin();
      __syncthreads();
      clear(sh);
      __syncthreads();
      row.each([&](float z, int i) {
        if (g.in(t, z, i)) {
          const int bin = g.bin_of(z, i);
          const unsigned w = mass ? (unsigned)(fminf(exp2_hw((z - zmax) * inv - edge(g, bin, zmax, inv)), 2.f) * 67108864.f) : 0u;
          atomicAdd(&sh.bin[bin], (u64)w | 1ull << 45);
        }
      });
      double all_w;
      find_bin(g, sh, zmax, inv, mass, by_mass, k, target, -1.f, all_w);
    }
    begun = false;
    const int bin = sh.at;
    if (tid == 0) sh.found_i = -1, sh.n = 0;
    __syncthreads();
    if (bin < 0) return t;
    const unsigned n = sh.here_n;
    if (n <= CAP) {
      if (tid < CAP && tid >= (int)n) some.key[tid] = 0, some.w[tid] = 0;
      row.each([&](float z, int i) {
        if (g.in(t, z, i) && g.bin_of(z, i) == bin) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < CAP) some.key[at] = order_key(z, i), some.w[at] = mass ? fixed(exp2_hw((z - zmax) * inv)) : 0;
        }
      });
      __syncthreads();
      if (tid < (int)n) {
        const u64 key = some.key[tid], own = some.w[tid];
        unsigned rank = 0;
        u64 w = 0;
        for (unsigned q0 = 0; q0 < n; q0 += 8)  // eight reads under way together
#pragma unroll
          for (unsigned q = 0; q < 8; ++q) {
            const u64 other = some.key[q0 + q], weight = some.w[q0 + q];
            rank += other > key;
            w += other > key ? weight : 0;
          }
        // (the bin's own sum has reached the target, so its last token has)
        const double cw = sh.above_w + bin_units(w), nw = sh.above_w + bin_units(w + own);
        if (by_mass ? (cw < target || !rank) && (nw >= target || rank == n - 1) : sh.above_n + rank == k - 1)
          sh.found_z = key_logit(key), sh.found_i = key_index(key), sh.run_w = nw;
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
    g.ties = g.hi == g.lo, g.first = false;
  }
}

struct Best { float s, z; int i; };
__device__ __forceinline__ void race(Best& b, float z, int i, float zmax, float inv, float u) {
  const float s = fmaxf((z - zmax) * inv - __builtin_amdgcn_logf(-__builtin_amdgcn_logf(fminf(u, 0.99999994f))), -FLT_MAX);
  if (s > b.s || (s == b.s && i < b.i)) b = {s, z, i};
}
// f(logit, index, uniform) for the tokens of every run of 16 bytes whose largest logit `maybe` takes.  The next run's logits and uniforms are asked for
// before this one's work.
template <typename T, typename M, typename F>
__device__ __forceinline__ void race_pass(const Row<T>& row, const float* u, M maybe, F f) {
  constexpr int VEC = Row<T>::VEC;
  const bool wide = (uintptr_t)u % 16 == 0;
  struct Run { uint4 v; float4 u[VEC / 4]; bool some; };
  auto fetch = [&](int q) {
    Run r;
    r.v = row.run(q);
    if (row.odd) r.v = Row<T>::mended(r.v);
    float most = NEG_INF;
    Row<T>::tokens(r.v, [&](float z, int) { most = fmaxf(most, z); });
    r.some = maybe(most);
    if (r.some) {
      const int first = q * VEC;
      if (wide && first + VEC <= row.V) {
#pragma unroll
        for (int e = 0; e < VEC / 4; ++e) r.u[e] = *reinterpret_cast<const float4*>(u + first + 4 * e);
      } else {
#pragma unroll
        for (int e = 0; e < VEC / 4; ++e)
          r.u[e] = make_float4(u[min(first + 4 * e, row.V - 1)], u[min(first + 4 * e + 1, row.V - 1)], u[min(first + 4 * e + 2, row.V - 1)],
                               u[min(first + 4 * e + 3, row.V - 1)]);
      }
    }
    return r;
  };
  int q = threadIdx.x;
  Run next{};
  if (q < row.n_vec) next = fetch(q);
#pragma unroll 1
  while (q < row.n_vec) {
    const int first = q * VEC;
    const Run now = next;
    q += NT;
    if (q < row.n_vec) next = fetch(q);
    if (now.some)
      Row<T>::tokens(now.v, [&](float z, int e) {
        const float4 x = now.u[e >> 2];
        f(z, first + e, (e & 3) == 0 ? x.x : (e & 3) == 1 ? x.y : (e & 3) == 2 ? x.z : x.w);
      });
  }
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
  row.n_lds = min(row.n_vec, a.row_bytes / 16);
  const int room = a.list;  // tokens of the list
  unsigned* const the_list = reinterpret_cast<unsigned*>(row_lds + row.n_lds);
  row.wide = (uintptr_t)row.p % 16 == 0;
  const float temp = a.temperature[r], top_p = a.top_p[r], min_p = fminf(a.min_p[r], 1.f);
  const int top_k = a.top_k[r];
  const bool greedy = !(temp > 0.f);
  clear(sh);
  if (tid < NC) sh.top[tid] = 0;
  if (tid == 0) sh.n = 0, sh.runs = 0, sh.odd = 0, sh.above_n = 0, sh.above_w = 0;
  float most = NEG_INF;
  bool odd = false;
  row.first([&](float z, int) {
    most = fmaxf(most, z);
    odd |= !(fabsf(z) <= FLT_MAX);
  });
  const float zmax = fminf(block_max(most, sh.part_a), Row<T>::TOP);
  if (odd) sh.odd = 1;
  const float by = greedy ? 1.f : fminf(fmaxf(1.0f / temp, 1e-30f), 1e30f), inv = LOG2E * by;
  const bool by_k = !greedy && top_k > 0 && top_k < a.V, by_p = !greedy && top_p < 1.f, small_k = by_k && top_k <= SMALL_K;
  Range range = {zmax, -FLT_MAX, fmaxf(zmax - DEPTH / inv, -FLT_MAX), false, 0, a.V, 0.f, 0, true};
  range.begin();
  const float coarse = range.c * ((float)NC / NB);
  if (small_k) atomicAdd(&sh.top[(int)fminf((zmax - fminf(most, Row<T>::TOP)) * coarse, (float)(NC - 1))], 1u);
  __syncthreads();
  row.odd = sh.odd;
  if (zmax == NEG_INF) {
    if (tid == 0) {
      a.token[g][r] = -1;
      if (a.logprob[g]) a.logprob[g][r] = NEG_INF;
    }
    return;
  }
  const float* u = a.u[g] + (size_t)r * a.ldu;
  const bool want_lse = a.logprob[g] != nullptr;
  float lse = 0.f;
  Best best = {NEG_INF, NEG_INF, 0x7fffffff};
  auto heavy = [&](float z) { return min_p <= 0.f || exp2_hw((z - zmax) * inv) >= min_p; };
  const bool both = by_k && by_p;
  const float p = fmaxf(top_p, 1e-30f);
  constexpr int VEC = Row<T>::VEC;
  // To the list, in two steps, in any order: the runs with some token that `maybe` belongs there (their numbers take the bins' place), then the
  // tokens of those that do.  One place is asked for per wave (a place per lane, of one counter, costs each lane a turn); as many runs at most as tokens.
  uint16_t* const run_list = reinterpret_cast<uint16_t*>(sh.bin);
  static_assert(WIDE_LIST * sizeof(uint16_t) <= sizeof(sh.bin), "the runs take the bins' place");
  auto place = [&](u64 hits, int first) { return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(hits >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)hits, (unsigned)first)); };
  auto places = [&](int& counter, int all) {
    int first = 0;
    if (place(~0ull, 0) == 0) first = atomicAdd(&counter, all);
    return __builtin_amdgcn_readfirstlane(first);
  };
  auto list_run = [&](bool maybe, int q) {
    const u64 hits = __ballot(maybe);
    if (!hits) return;
    const int at = place(hits, places(sh.runs, __popcll(hits)));
    if (maybe && at < room) run_list[at] = (uint16_t)q;
  };
  auto list_tokens = [&](auto in) {
    __syncthreads();
    const int n_runs = min(sh.runs, room);
#pragma unroll 1
    for (int r = tid; r < n_runs; r += NT) {
      const int q = (int)run_list[r];
      uint4 v = row.run(q);
      if (row.odd) v = Row<T>::mended(v);
      u64 hits[VEC];
      bool is[VEC];
      int all = 0;
      Row<T>::tokens(v, [&](float z, int e) {
        is[e] = in(z);
        hits[e] = __ballot(is[e]), all += __popcll(hits[e]);
      });
      int first = places(sh.n, all);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int at = place(hits[e], first);
        if (is[e] && at < room) the_list[at] = (unsigned)(q * VEC + e);
        first += __popcll(hits[e]);
      }
    }
    __syncthreads();
  };

  double target = 0;
  bool lse_left = want_lse, drawn = false, begun = false;
  unsigned n = room + 1;  // tokens in the list that hold all that can be kept, or none such
  float bins = (float)NB;  // of the first round's that matter
  if (greedy) {
    row.each([&](float z, int i) {
      if (want_lse) lse += exp2_hw((z - zmax) * LOG2E);
      if (z == zmax && i < best.i) best = {0.f, z, i};
    });
    drawn = true;
  } else if (!by_k && !by_p && min_p <= 0.f) {
    race_pass(row, u, [](float) { return true; }, [&](float z, int i, float x) {
      if (want_lse) lse += exp2_hw((z - zmax) * LOG2E);
      if (z > NEG_INF) race(best, z, i, zmax, inv, x);
    });
    drawn = true;
  } else if (small_k || min_p > 0.f) {
    // Tokens at or above a cut go to the list, in the pass that sums the weights.  What min_p leaves is known beforehand (with room for the
    // rounding of w; it is looked at exactly in the end), and of the threads' largest logits, the top_k-th has top_k tokens at or above it.
    float by_rank = __builtin_inff();
    if (small_k) {
      const uint4 c4 = reinterpret_cast<const uint4*>(sh.top)[tid & 63];
      const int sum4 = (int)(c4.x + c4.y + c4.z + c4.w);
      int upto = sum4;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(upto, d);
        if ((tid & 63) >= d) upto += up;
      }
      // the bin that reaches top_k, in the one lane whose bins do
      const unsigned b0 = (unsigned)(upto - sum4) + c4.x, b1 = b0 + c4.y, b2 = b1 + c4.z, k = (unsigned)top_k;
      const int at = 4 * (tid & 63) + (int)(b0 < k) + (int)(b1 < k) + (int)(b2 < k);
      const int bin = __builtin_amdgcn_readlane(at, __ffsll(__ballot(upto >= top_k)) - 1);
      if (bin < NC - 1) by_rank = (float)(bin + 1);
    }
    const float by_min = min_p > 0.f ? (1e-5f - 1.00001f * __builtin_amdgcn_logf(min_p)) / inv * coarse * 1.00001f : __builtin_inff();
    const bool whole = by_min <= by_rank;  // the list gets all that can be kept
    const float to = fminf(by_min, by_rank);
    const float least = fmaxf(zmax - to / coarse * 1.0001f, -FLT_MAX);
    const bool more = want_lse && !(by_p && inv == LOG2E);  // at temperature 1 it is the sum of all weights
    float mass = 0.f;
    row.runs([&](const uint4& v, int q) {
      float most = NEG_INF;
      Row<T>::tokens(v, [&](float z, int) { most = fmaxf(most, z); });
      if (by_p) Row<T>::tokens(v, [&](float z, int) { mass += exp2_hw((z - zmax) * inv); });
      if (more) Row<T>::tokens(v, [&](float z, int) { lse += exp2_hw((z - zmax) * LOG2E); });
      list_run(most >= least, q);
    });
    if (want_lse && !more) lse = mass;
    lse_left = false;
    mass = wave_sum(mass);
    if ((tid & 63) == 0) sh.part_a[tid >> 6] = mass;
    list_tokens([&](float z) { return z >= least; });
    double total = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) total += (double)sh.part_a[i];
    target = p * (total * BIN_ONE);
    n = sh.runs > room ? room + 1 : sh.n;
    if (n > (unsigned)room || !(n >= (unsigned)top_k || (whole && !both))) {  // too many, or not all that top_k keeps (or top_p's sum is over)
      // where the cut holds all that the rules look at, what is below its bins need not be counted again
      if (!by_k || n >= (unsigned)top_k) bins = fminf(bins, ceilf(to * ((float)NB / NC)) + 1.f);
      n = room + 1;
      __syncthreads();
      clear(sh);
      if (tid == 0) sh.n = 0, sh.runs = 0;
      __syncthreads();
    }
  }
  if (!drawn && n > (unsigned)room) {
    // the first round, over all tokens that can be drawn
    const float step = inv / range.c;  // log2 of the weights of two edges
    const bool lse_here = lse_left && !(by_p && inv == LOG2E);  // at temperature 1 it is the sum of all weights
    row.runs([&](const uint4& v, int) {
      Row<T>::tokens(v, [&](float z, int) {
        const float d = zmax - z, t = d * range.c, bin = truncf(fminf(t, (float)(NB - 1)));
        const unsigned w = by_p ? (unsigned)fminf(exp2_hw(fmaf(bin - t, step, 26.f)), 134217728.f) : 0u;
        if (bin < bins) atomicAdd(&sh.bin[(int)bin], (u64)(z > NEG_INF ? 1u << 13 : 0u) << 32 | w);
      });
      if (lse_here) Row<T>::tokens(v, [&](float z, int) { lse += exp2_hw((z - zmax) * LOG2E); });
    });
    // both rules end at or before where the first one does: the k-th token, or without top-k the share of all mass
    double all_w;
    target = find_bin(range, sh, zmax, inv, by_p, !by_k, (unsigned)top_k, target, by_k || bins < (float)NB ? -1.f : p, all_w);
    if (lse_left && !lse_here && tid == 0) lse = (float)(all_w * (1.0 / BIN_ONE));
    begun = true;
    if (sh.at >= 0) {
      // to the list: all tokens up to the bin's end, where that many fit; otherwise those of the bin, where they do
      n = sh.above_n + sh.here_n <= (unsigned)room ? sh.above_n + sh.here_n : room + 1;
      const unsigned here = sh.here_n;
      const float from = n <= (unsigned)room ? -1.f : (float)sh.at, to = sh.at == NB - 1 ? __builtin_inff() : (float)(sh.at + 1);
      if (here <= (unsigned)room) {
        auto in = [&](float z) {
          const float at = fminf((zmax - z) * range.c, FLT_MAX);
          return z > NEG_INF && at >= from && at < to;
        };
        row.runs([&](const uint4& v, int q) {
          bool some = false;
          if (from < 0.f) {
            float most = NEG_INF;
            Row<T>::tokens(v, [&](float z, int) { most = fmaxf(most, z); });
            some = in(most);
          } else {
            Row<T>::tokens(v, [&](float z, int) { some |= in(z); });
          }
          list_run(some, q);
        });
        list_tokens(in);
      }
    }
  }
  if (!drawn && n <= FEW) {  // a thread per token
    Some& some = *reinterpret_cast<Some*>(sh.bin);
    float z = NEG_INF, x = 0.f;
    int i = 0, rank = 0;
    u64 key = 0, own = 0, before = 0;
    if (tid < (int)n) {
      i = (int)the_list[tid], z = row.at(i), x = u[i];
      key = order_key(z, i), own = fixed(exp2_hw((z - zmax) * inv));
    }
    if (tid < FEW) some.key[tid] = key, some.w[tid] = 0;  // 0 behind the last one
    __syncthreads();
    if (tid < (int)n) {
      for (unsigned q0 = 0; q0 < n; q0 += 16)  // sixteen reads under way together
#pragma unroll
        for (unsigned q = 0; q < 16; ++q) rank += some.key[q0 + q] > key;
      some.w[rank] = own;
    }
    if (by_p) {  // weights in order, then their sums, by one wave
      __syncthreads();
      if (tid < 64) {
        const u64 w0 = some.w[2 * tid], w1 = some.w[2 * tid + 1];
        u64 sum = w0 + w1;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const u64 up = __shfl_up(sum, d);
          if (tid >= d) sum += up;
        }
        some.key[2 * tid] = sum - w0 - w1, some.key[2 * tid + 1] = sum - w1;
        if (both && (top_k - 1) >> 1 == tid) sh.run_w = bin_units((top_k & 1) ? sum - w1 : sum);
      }
      __syncthreads();
      if (both) target = p * sh.run_w;
      if (tid < (int)n) before = some.key[rank];
    }
    if (tid < (int)n && (!by_k || rank < top_k) && (!by_p || !rank || bin_units(before) < target) && heavy(z)) race(best, z, i, zmax, inv, x);
  } else if (!drawn) {
    // the rules one after the other, the first one over the list or the whole row (where its bin's tokens did not fit)
    const bool listed = n <= (unsigned)room;
    Last t = {-FLT_MAX, 0x7fffffff};
    Tokens<T> tokens = {row, the_list, (int)n, listed};
    if (begun && !listed && sh.at >= 0 && sh.here_n <= (unsigned)room) tokens.n = (int)sh.here_n, tokens.listed = true;
    const int rules = (int)by_k + (int)by_p;
#pragma unroll 1
    for (int rule = 0; rule < rules; ++rule) {
      if (rule) {
        tokens.n = (int)n, tokens.listed = listed;
        double total = sh.run_w;
        if (sh.found_i < 0) {  // fewer than k tokens can be drawn: all of them are kept
          double w = 0, x_w;
          unsigned x_n;
          tokens.each([&](float z, int) { w += (double)exp2_hw((z - zmax) * inv); });
          __syncthreads();
          double* const sums = reinterpret_cast<double*>(sh.bin);
          sums[tid] = w;
          __syncthreads();
          for (int i = NS + tid; tid < NS && i < NT; i += NS) w += sums[i];
          block_scan(0, w * BIN_ONE, x_n, x_w, total, sh);
        }
        target = p * total;
        __syncthreads();
        if (tid == 0) sh.above_n = 0, sh.above_w = 0;
      }
      t = find_last(tokens, sh, range, begun && !rule, t, zmax, inv, rule || !by_k, (unsigned)top_k, target, by_p);
    }
    if (listed) {
#pragma unroll 1
      for (int e0 = tid; e0 < (int)n; e0 += 4 * NT) {  // four gathers under way together
        int i[4];
        float z[4], x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) i[e] = e0 + e * NT < (int)n ? (int)the_list[e0 + e * NT] : -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = i[e] >= 0 ? row.at(i[e]) : NEG_INF, x[e] = i[e] >= 0 ? u[i[e]] : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (z[e] > NEG_INF && kept(t, z[e], i[e]) && heavy(z[e])) race(best, z[e], i[e], zmax, inv, x[e]);
      }
    } else {
      race_pass(row, u, [&](float z) { return z >= t.z; }, [&](float z, int i, float x) {
        if (z > NEG_INF && kept(t, z, i) && heavy(z)) race(best, z, i, zmax, inv, x);
      });
    }
  }
  auto join = [&](int d) {
    const Best o = {__shfl_xor(best.s, d), __shfl_xor(best.z, d), __shfl_xor(best.i, d)};
    if (o.s > best.s || (o.s == best.s && o.i < best.i)) best = o;
  };
  if (__any(best.s > NEG_INF)) {
#pragma unroll
    for (int d = 32; d; d >>= 1) join(d);
  }
  lse = wave_sum(lse);
  __syncthreads();
  if ((tid & 63) == 0) sh.part_a[tid >> 6] = best.s, sh.part_i[tid >> 6] = best.i, sh.part_z[tid >> 6] = best.z, sh.part_b[tid >> 6] = lse;
  __syncthreads();
  if (tid < 64) {
    constexpr int NW = NT / 64;
    best = {sh.part_a[tid % NW], sh.part_z[tid % NW], sh.part_i[tid % NW]};
#pragma unroll
    for (int d = NW / 2; d; d >>= 1) join(d);
    if (tid == 0) {
      a.token[g][r] = best.i;
      if (want_lse) {
        lse = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) lse += sh.part_b[i];
        a.logprob[g][r] = best.z - zmax - __builtin_amdgcn_logf(lse) * LN2;
      }
    }
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
  hipError_t e = hipFuncSetAttribute((const void*)sample_kernel<float>, hipFuncAttributeMaxDynamicSharedMemorySize, ROW_BYTES + 4 * LIST);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)sample_kernel<bf16_t>, hipFuncAttributeMaxDynamicSharedMemorySize, ROW_BYTES + 4 * LIST);
}

hipError_t launch_sample(const SampleArgs& args, hipStream_t s) {
  SampleArgs a = args;
  const size_t esize = a.dtype == GEMM_F32 ? 4 : 2, row = ((size_t)a.V * esize + 15) / 16 * 16;
  const bool fits = row <= ROW_BYTES;
  a.list = fits ? LIST : WIDE_LIST;
  a.row_bytes = fits ? (int)row : WIDE_ROW_BYTES;
  const unsigned lds = (unsigned)(a.row_bytes + 4 * a.list);
  const dim3 grid(a.rows, a.G);
  if (a.dtype == GEMM_F32) hipLaunchKernelGGL((sample_kernel<float>), grid, dim3(NT), lds, s, a);
  else hipLaunchKernelGGL((sample_kernel<bf16_t>), grid, dim3(NT), lds, s, a);
  return hipGetLastError();
}

}  // namespace hydra
