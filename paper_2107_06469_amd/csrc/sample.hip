// Drawing one token per row of logits with temperature, top-k, top-p and min-p from given uniforms.
//   Tokens in order: larger logit first, the lower index first among equals.  Kept are, of w_i = exp((z_i - max z) / T):
//     the first k (top_k > 0);  of those the shortest run from the first on whose sum of w reaches top_p times the sum of all of them (top_p < 1);
//     of those the ones with w_i >= min_p.  All three are runs from the first token on, so that "kept" is one comparison with a last (logit, index).
//   token = argmax over kept of z_i / T - log(-log u_i), the lowest index first: with u uniform, a draw with probabilities proportional to w_i.
//   T <= 0: the largest logit.  logprob = z_token - log sum_i exp z_i over all tokens, at temperature 1.
//   A logit of -inf or NaN is never drawn, +inf counts as the largest float; without a token that can be drawn: -1 and -inf.
// A row is one workgroup's.  The last kept token is found by histograms: 2048 bins over the range of logits in question hold counts and sums
// of w (in fixed point, 2^-44, so that no order of additions matters); the bin where the count or sum is reached is the next range, until
// what it holds fits a list that is ranked directly.  Equal logits are told apart by histograms over their indices.
#include <float.h>

#include "kernels.h"
#include "wave_math.h"

namespace hydra {
namespace {

constexpr int NT = 1024, NB = 2048, CAP = 256;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_inff();
typedef unsigned long long u64;

struct Last { float z; int i; };  // the last kept token: kept are larger logits, and equal ones up to its index
__device__ __forceinline__ bool kept(const Last& t, float z, int i) { return z > t.z || (z == t.z && i <= t.i); }

__device__ __forceinline__ float logit(float z) { return z == z ? fminf(z, FLT_MAX) : NEG_INF; }
__device__ __forceinline__ float load(const float* p) { return logit(*p); }
__device__ __forceinline__ float load(const bf16_t* p) { return logit(__uint_as_float((uint32_t)*p << 16)); }

struct Shared {
  unsigned count[NB];
  u64 mass[NB];
  float list_z[CAP];
  int list_i[CAP];
  u64 list_w[CAP];
  float part_a[NT / 64], part_b[NT / 64];
  int part_i[NT / 64];
  unsigned part_n[NT / 64];
  u64 part_w[NT / 64];
  int n, bin, found_i;
  unsigned above_n;
  u64 above_w, total_w;
  float found_z;
};

// The row's elements: held in registers (element 1024 k + thread), or read again where they do not fit.
template <typename T, int EPT>
struct Row {
  float z[EPT ? EPT : 1];
  const T* p;
  int V;
  template <typename F>
  __device__ __forceinline__ void each(F f) {
    if constexpr (EPT > 0) {
#pragma unroll
      for (int k = 0; k < EPT; ++k) f(z[k], k * NT + (int)threadIdx.x);
    } else {
      for (int i = threadIdx.x; i < V; i += NT) f(load(p + i), i);
    }
  }
};

__device__ __forceinline__ float block_max(float v, float* part) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = part[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) r = fmaxf(r, part[i]);
  return r;
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

// The first bin at which above + the bins' sum so far reaches the target, by count or by mass; sh.bin = -1 where none does.  sh.above_* then are the
// sums before it.
__device__ __forceinline__ void find_bin(Shared& sh, bool by_mass, unsigned k, u64 target) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __syncthreads();
  const unsigned n0 = sh.count[2 * tid], n1 = sh.count[2 * tid + 1];
  const u64 w0 = sh.mass[2 * tid], w1 = sh.mass[2 * tid + 1];
  unsigned n = n0 + n1;
  u64 w = w0 + w1;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned pn = __shfl_up(n, d);
    const u64 pw = __shfl_up(w, d);
    if (lane >= d) n += pn, w += pw;
  }
  if (lane == 63) sh.part_n[wave] = n, sh.part_w[wave] = w;
  const unsigned an = sh.above_n;
  const u64 aw = sh.above_w;
  __syncthreads();
  if (tid == 0) sh.bin = -1;
  n += an, w += aw;
  for (int i = 0; i < wave; ++i) n += sh.part_n[i], w += sh.part_w[i];
  __syncthreads();
  // sums through the end of bin 2 tid, and through 2 tid + 1
  const unsigned na = n - n1;
  const u64 wa = w - w1;
  const bool here0 = by_mass ? wa - w0 < target && wa >= target : na - n0 < k && na >= k;
  const bool here1 = by_mass ? wa < target && w >= target : na < k && n >= k;
  if (here0) sh.bin = 2 * tid, sh.above_n = na - n0, sh.above_w = wa - w0;
  if (here1) sh.bin = 2 * tid + 1, sh.above_n = na, sh.above_w = wa;
  __syncthreads();
}
__device__ __forceinline__ void clear(Shared& sh) {
  __syncthreads();
  for (int i = threadIdx.x; i < NB; i += NT) sh.count[i] = 0, sh.mass[i] = 0;
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
}

// The last token of the run that reaches k tokens or the target mass, among those kept by `t`; t itself where nothing does.  sh.total_w: the mass
// of the run, where it is found.  inv: log2(e) / T.
template <typename R>
__device__ __forceinline__ Last find_last(R& row, Shared& sh, Last t, float zmax, float zmin, float inv, bool by_mass, unsigned k, u64 target, bool mass) {
  const int tid = threadIdx.x;
  auto weight = [&](float z) { return fixed(__builtin_amdgcn_exp2f((z - zmax) * inv)); };
  float hi = zmax, lo = fmaxf(zmin, t.z);
  float low = fmaxf(lo, hi - 24.f * 1.4426950408889634f / inv);  // the bins end here at first: what is below goes to the last one
  __syncthreads();
  if (tid == 0) sh.above_n = 0, sh.above_w = 0, sh.found_i = -1;
  bool ties = false;  // all that is left has the logit hi: bins of indices
  int i_lo = 0, i_n = row.V;
  while (true) {  // a round takes the largest logit of its range (ties: the other bins' indices) out of the next one
    clear(sh);
    const float c = fminf((float)NB / (hi - low), FLT_MAX);
    const unsigned per = (unsigned)(i_n + NB - 1) / NB;
    auto in = [&](float z, int i) { return z <= hi && z >= lo && kept(t, z, i) && (!ties || (i >= i_lo && i < i_lo + i_n)); };
    auto bin_of = [&](float z, int i) { return ties ? (int)((unsigned)(i - i_lo) / per) : z == hi ? 0 : (int)fminf(fmaxf((hi - z) * c, 1.f), (float)(NB - 1)); };
    row.each([&](float z, int i) {
      if (in(z, i)) {
        const int bin = bin_of(z, i);
        atomicAdd(&sh.count[bin], 1u);
        if (mass) atomicAdd(&sh.mass[bin], weight(z));
      }
    });
    find_bin(sh, by_mass, k, target);
    const int bin = sh.bin;
    if (bin < 0) return t;
    const unsigned n = sh.count[bin];
    if (n <= CAP) {
      row.each([&](float z, int i) {
        if (in(z, i) && bin_of(z, i) == bin) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < CAP) sh.list_z[at] = z, sh.list_i[at] = i, sh.list_w[at] = mass ? weight(z) : 0;
        }
      });
      __syncthreads();
      if (tid < (int)n) {
        const float z = sh.list_z[tid];
        const int i = sh.list_i[tid];
        unsigned before = sh.above_n;
        u64 w = sh.above_w;
        for (unsigned q = 0; q < n; ++q) {
          const float zq = sh.list_z[q];
          const int iq = sh.list_i[q];
          if (zq > z || (zq == z && iq < i)) ++before, w += sh.list_w[q];
        }
        const u64 own = sh.list_w[tid];
        if (by_mass ? w < target && w + own >= target : before == k - 1) sh.found_z = z, sh.found_i = i, sh.total_w = w + own;
      }
      __syncthreads();
      return sh.found_i < 0 ? t : Last{sh.found_z, sh.found_i};
    }
    if (ties) {
      i_lo += bin * per, i_n = min((int)per, i_n - bin * (int)per);
      continue;
    }
    float most = NEG_INF, least = NEG_INF;  // the range of what is in the bin (the smaller one with its sign turned)
    row.each([&](float z, int i) {
      if (in(z, i) && bin_of(z, i) == bin) most = fmaxf(most, z), least = fmaxf(least, -z);
    });
    hi = block_max(most, sh.part_a);
    lo = low = -block_max(least, sh.part_b);
    ties = hi == lo;
  }
}

template <typename T, int EPT>
__global__ __launch_bounds__(NT) void sample_kernel(const SampleArgs a) {
  __shared__ Shared sh;
  const int g = blockIdx.y, r = blockIdx.x, tid = threadIdx.x;
  Row<T, EPT> row;
  row.V = a.V;
  row.p = static_cast<const T*>(a.z[g]) + (size_t)r * a.ldz;
  const float temp = a.temperature[r], top_p = a.top_p[r], min_p = fminf(a.min_p[r], 1.f);
  const int top_k = a.top_k[r];
  if constexpr (EPT > 0) {
#pragma unroll
    for (int k = 0; k < EPT; ++k) {
      const int i = k * NT + tid;
      row.z[k] = i < a.V ? load(row.p + i) : NEG_INF;
    }
  }
  const bool greedy = !(temp > 0.f);
  float most = NEG_INF, least = NEG_INF;
  row.each([&](float z, int) {
    most = fmaxf(most, z);
    least = fmaxf(least, z == NEG_INF ? NEG_INF : -z);
  });
  const float zmax = block_max(most, sh.part_a), zmin = -block_max(least, sh.part_b);
  if (zmax == NEG_INF) {
    if (tid == 0) {
      a.token[g][r] = -1;
      if (a.logprob[g]) a.logprob[g][r] = NEG_INF;
    }
    return;
  }
  float lse = 0.f;
  if (a.logprob[g]) {
    row.each([&](float z, int) { lse += __builtin_amdgcn_exp2f((z - zmax) * LOG2E); });
    lse = block_sum(lse, sh.part_a);
  }
  const float by = greedy ? 1.f : fminf(fmaxf(1.0f / temp, 1e-30f), 1e30f), inv = LOG2E * by;
  Last t = {zmin, 0x7fffffff};
  if (greedy) {
    t.z = zmax;
  } else {
    const bool by_k = top_k > 0 && top_k < a.V, by_p = top_p < 1.f;
    bool have = false;
    u64 total = 0;
    if (by_k) {
      t = find_last(row, sh, t, zmax, zmin, inv, false, (unsigned)top_k, 0, by_p);
      have = sh.found_i >= 0;
      total = sh.total_w;
    }
    if (by_p) {
      if (!have) {
        u64 w = 0;
        row.each([&](float z, int) { w += fixed(__builtin_amdgcn_exp2f((z - zmax) * inv)); });
#pragma unroll
        for (int d = 32; d; d >>= 1) w += __shfl_xor(w, d);
        __syncthreads();
        if ((tid & 63) == 0) sh.part_w[tid >> 6] = w;
        __syncthreads();
        total = 0;
        for (int i = 0; i < NT / 64; ++i) total += sh.part_w[i];
      }
      const double want = __builtin_ceil((double)fmaxf(top_p, 0.f) * (double)total);
      t = find_last(row, sh, t, zmax, zmin, inv, true, 0, want < 1.0 ? 1ull : (u64)want, true);
    }
  }
  // the race among the kept
  float best = NEG_INF, best_z = NEG_INF;
  int at = 0x7fffffff;
  const float* u = a.u[g] + (size_t)r * a.ldu;
  row.each([&](float z, int i) {
    if (z > NEG_INF && kept(t, z, i) && (greedy || __builtin_amdgcn_exp2f((z - zmax) * inv) >= min_p)) {
      const float s = greedy ? z : fmaxf((z - zmax) * by - logf(-logf(fminf(u[i], 0.99999994f))), -FLT_MAX);
      if (s > best || (s == best && i < at)) best = s, best_z = z, at = i;
    }
  });
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float s = __shfl_xor(best, d), z = __shfl_xor(best_z, d);
    const int i = __shfl_xor(at, d);
    if (s > best || (s == best && i < at)) best = s, best_z = z, at = i;
  }
  __syncthreads();
  if ((tid & 63) == 0) sh.part_a[tid >> 6] = best, sh.part_b[tid >> 6] = best_z, sh.part_i[tid >> 6] = at;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < NT / 64; ++i)
      if (sh.part_a[i] > best || (sh.part_a[i] == best && sh.part_i[i] < at)) best = sh.part_a[i], best_z = sh.part_b[i], at = sh.part_i[i];
    a.token[g][r] = at;
    if (a.logprob[g]) a.logprob[g][r] = best_z - zmax - logf(lse);
  }
}

template <typename T>
void run_sample(const SampleArgs& a, hipStream_t s) {
  const dim3 grid(a.rows, a.G);
  if (a.V <= 8 * NT) hipLaunchKernelGGL((sample_kernel<T, 8>), grid, dim3(NT), 0, s, a);
  else if (a.V <= 32 * NT) hipLaunchKernelGGL((sample_kernel<T, 32>), grid, dim3(NT), 0, s, a);
  else hipLaunchKernelGGL((sample_kernel<T, 0>), grid, dim3(NT), 0, s, a);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.G < 1 || a.G > MAXG || a.rows < 1 || a.V < 1 || a.V > (1 << 24) || a.ldz < a.V || a.ldu < a.V) return hipErrorInvalidValue;
  if (a.dtype == GEMM_F32) run_sample<float>(a, s);
  else run_sample<bf16_t>(a, s);
  return hipGetLastError();
}

}  // namespace hydra
