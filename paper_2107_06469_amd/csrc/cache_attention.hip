// Attention of new tokens over a paged cache of 8-bit codes (kv_cache.hip writes it).
//   s[i,t] = (q_i . k_t) * scale,  k_t = code_t * s_page;  t < length, and t <= position of i under a causal mask;  p = softmax over t;
//   o_i = sum_t p[i,t] v_t,  lse_i = log sum_t exp s[i,t];  a row that sees nothing: o = 0, lse = -inf.
// The rows of one key/value head are all its query heads of all tokens of the call, (token, head) in that order, so that every code is read once
// for all of them.
//
// Codes never leave registers between memory and the matrix cores.  Both products run on v_mfma_f32_16x16x32_f16: codes are exact in f16 (11
// bits), p in f16 is rounded to 2^-12, finer than bf16 would, and a query row, bf16, is exact in f16 once the power of two of its largest
// element is taken out (elements below 2^-17 of that are rounded to 2^-25 of it, half of what an fp32 sum with it may lose anyway).
//   S^T[t,i] = K Q^T:  lane l supplies row t = l%16 of K, 16 bytes at a time as they lie in memory, and gets column i = l%16, rows 4(l/16) + e
//   O^T[d,i] += V^T P^T: the accumulators of two 16-key tiles are, in that order, the B operand (k index = accumulator row), and the A operand is,
//     for d = W (l%16) + c (W = DH/16 bytes, one load), byte c of the 8 keys' words: one byte permutation brings two keys' codes together.
// A page's scale of keys multiplies its scores; that of its values, in units of the largest one met so far, is in the exponent of its weights, whose own sum
// takes it back.  A row's maximum is that of what is in the exponents, so that f16, which holds weights down to 2^-39 of the largest, measures them by
// what a page gives to the row, however small the values of the pages that the row looks at (down to 2^-64 of the largest; smaller scales
// count as that).  Maxima, sums, scores and accumulators are fp32.
//
// Bound by HBM where there are keys to read, 2 DH bytes each and head: 2 x 64 sequences of up to 2048 tokens over 8 heads of 128 (406 MB) in 76 us,
// 5.3 TB/s, where the loads alone of this kernel take 70; 8 of up to 32768 (385 MB) in 72.  One sequence of 513 tokens takes 9, nearly all of it
// latency: lengths and pages, codes, the join of the waves.
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "wave_math.h"

namespace hydra {
namespace {

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_BIG = -1.0e30f;
constexpr float P_LOG2 = 15.f, P_ONE = 32768.f;  // a weight of 1 in f16
constexpr float LEAST_UNITS = 0x1p-64f, SUM_LOG2 = 96.f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const f16x2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// An int8 code c with its sign bit turned over is u = 128 + c.  In a half by itself u is a (subnormal) f16 number, u 2^-24, which the matrix
// cores take as any other.  What the 128 add to a score is known beforehand: its accumulator begins there.  From values they are taken off at once (c 2^-24 is
// exact, too): taken off a sum they would leave 2^-17 of the largest code in columns that are small.
constexpr float U_ONE = 16777216.f;  // 2^24
template <int KIND>
__device__ __forceinline__ uint32_t turned(uint32_t w) { return KIND == CACHE_INT8 ? w ^ 0x80808080u : w; }
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_halves(uint32_t w) {
  return __builtin_bit_cast(uint32_t, (f16x2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
}
// eight codes in a row: their values, or of int8 u 2^-24
template <int KIND>
__device__ __forceinline__ uint4 wide8(uint32_t lo, uint32_t hi) {
  if (KIND == CACHE_E4M3) return make_uint4(e4m3_halves<false>(lo), e4m3_halves<true>(lo), e4m3_halves<false>(hi), e4m3_halves<true>(hi));
  lo = turned<KIND>(lo), hi = turned<KIND>(hi);
  return make_uint4(__builtin_amdgcn_perm(0, lo, 0x0c010c00u), __builtin_amdgcn_perm(0, lo, 0x0c030c02u), __builtin_amdgcn_perm(0, hi, 0x0c010c00u),
                    __builtin_amdgcn_perm(0, hi, 0x0c030c02u));
}
// bytes C and C + 1 (C even) of two keys' (turned) words -> {key 0, key 1} of column C and of column C + 1, of int8 times 2^-24
template <int KIND, int C>
__device__ __forceinline__ uint2 columns2(uint32_t k0, uint32_t k1) {
  if (KIND == CACHE_E4M3) {
    const uint32_t w = __builtin_amdgcn_perm(k1, k0, (unsigned)C | (4u + C) << 8 | (1u + C) << 16 | (5u + C) << 24);
    return make_uint2(e4m3_halves<false>(w), e4m3_halves<true>(w));
  }
  auto code = [&](uint32_t sel) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(k1, k0, sel)) + __builtin_bit_cast(f16x2, 0x80808080u));  // - 128 2^-24
  };
  return make_uint2(code(0x0c000c00u | C | (4u + C) << 16), code(0x0c000c00u | (C + 1) | (5u + C) << 16));
}

// max over the four lanes that share l%16
__device__ __forceinline__ float quarter_max(float v) {
  float2 p = wave_swap32(v);
  v = fmaxf(p.x, p.y);
  p = wave_swap16(v);
  return fmaxf(p.x, p.y);
}
__device__ __forceinline__ float quarter_sum(float v) {
  float2 p = wave_swap32(v);
  v = p.x + p.y;
  p = wave_swap16(v);
  return p.x + p.y;
}

__device__ __forceinline__ float sum8(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f16x2 h = __builtin_bit_cast(f16x2, w[i]);
    s += (float)h.x + (float)h.y;
  }
  return s;
}
// A page's scale of values in units of the largest; where there is none, 1.
__device__ __forceinline__ float in_units(float scale, float unit) { return unit > 0.f ? fmaxf(scale / unit, LEAST_UNITS) : 1.f; }
// The largest scale of values has grown from `unit` to `now`: what a row's accumulators are to be multiplied by.  Its maximum, which is in these units, goes
// down with them, so that weights to come are measured by what the row has got so far, as far as its sum (`sum`, of which the lane holds l) stays a number.
__device__ __forceinline__ float other_unit(float unit, float now, float sum, float& m, float& l) {
  const float grown = unit > 0.f ? fminf(__builtin_amdgcn_logf(now) - __builtin_amdgcn_logf(unit), 250.f) : 250.f;
  const float down = fminf(grown, fmaxf(SUM_LOG2 - __builtin_amdgcn_logf(sum), 0.f));
  m -= down, l *= fast_exp2(down);
  return unit > 0.f ? fast_exp2(down - grown) : 0.f;
}
// Codes that one workgroup reads once: past the caches' order of use.
__device__ __forceinline__ uint4 once16(const uint8_t* p) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}
__device__ __forceinline__ uint2 once8(const uint8_t* p) {
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p)));
}
__device__ __forceinline__ int lane_int(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float lane_float(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

struct CacheAttnPlan {
  int n_split, chunk;  // runs of keys, keys in one (a multiple of 128)
  int n_rt;            // 16-row tiles, or the prompt kernel's blocks, of the sequence with the most rows
  int page_log2;
  int waves;           // of a workgroup
  bool prompt;         // cache_prompt_kernel, 32 rows a wave; else cache_attn_kernel
};

// NW waves share a run of keys, 32 at a time in turn, each with its own maximum, sum and accumulators; they are joined through LDS.  A tile of V
// is read past the caches' order of use, one of K through it (its rows are taken by two loads each): the other way round, 8 sequences of 32768
// tokens take 78..85 us (V cached) and 82 (K past it) instead of 77.
// blockIdx: x sequence and key/value head, y run of keys and row tile, z model.
template <int DH, int NW>
constexpr int attn_lds() { return NW * 16 * (DH + 4) * 4 + NW * 16 * 8; }
template <int KIND, int DH, int NW>
__global__ __launch_bounds__(NW * 64) void cache_attn_kernel(const CacheAttnArgs a, const CacheAttnPlan pl) {
  constexpr int W = DH / 16, NK = DH / 32, NL = DH / 64;  // bytes of a V load; k steps of a score; K loads of 16 bytes per lane
  extern __shared__ __attribute__((aligned(16))) float w_o[];  // [NW][16][DH + 4], then the maxima and sums [NW][16]
  float2* const w_ml = reinterpret_cast<float2*>(w_o + NW * 16 * (DH + 4));
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, gq = lane >> 4;
  const int g = blockIdx.z, b = blockIdx.x / c.HKV, h = blockIdx.x - b * c.HKV;
  const int split = blockIdx.y / pl.n_rt, rt = blockIdx.y - split * pl.n_rt;
  const int t_lo = split * pl.chunk;
  // lane i knows page i of a segment of 64 pages (the first one's numbers come with the lengths, whatever these are)
  auto page_at = [&](int seg) {
    const int i = (seg >> pl.page_log2) + lane;
    return i < c.max_pages ? c.table[(size_t)b * c.max_pages + i] : -1;
  };
  const int first_pages = page_at(t_lo);
  const CacheSeq sq = cache_seq(c, b);
  const int share = a.H / c.HKV, rows = sq.n * share, first = rt * 16;
  if (first >= rows) return;
  const int all = a.causal ? max(sq.pos0 + (min(first + 16, rows) - 1) / share + 1, 0) : sq.len;  // keys that the tile's last row sees
  const int t_hi = min(t_lo + pl.chunk, all);
  auto page_of = [&](int seg, int id) { return seg + (lane << pl.page_log2) < t_hi && (unsigned)id < (unsigned)c.n_pages ? id : -1; };
  int id = page_of(t_lo, first_pages);
  // this lane's row
  const bool have = first + r < rows;
  const int row = have ? first + r : first, j = row / share, hq = h * share + row - j * share;
  const int sees = have ? (a.causal ? max(sq.pos0 + j + 1, 0) : sq.len) : 0;  // keys
  const int free = min(t_hi, a.causal ? sq.pos0 + first / share + 1 : sq.len);  // keys that every row of the tile sees
  uint4 q_raw[NK];
  {
    const bf16_t* q = a.q[g] + (size_t)(sq.row0 + j) * a.ld_q + (size_t)hq * DH;
#pragma unroll
    for (int k = 0; k < NK; ++k) q_raw[k] = *reinterpret_cast<const uint4*>(q + ((k >> 1) * 4 + gq) * 16 + (k & 1) * 8);
  }
  // one 32-key tile
  struct Tile { uint4 k[2][NL]; uint2 v[2][4]; };
  const int page_mask = c.page - 1;
  auto fetch = [&](Tile& x, int seg, int t) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int ts = t + 16 * s, pid = max(lane_int(id, (ts - seg) >> pl.page_log2 & 63), 0);
      const size_t at = (size_t)pid * c.page_bytes + ((size_t)h * c.page + (ts & page_mask)) * DH;
      const uint8_t* kp = c.k[g] + at + r * DH + gq * 16;
#pragma unroll
      for (int i = 0; i < NL; ++i) x.k[s][i] = *reinterpret_cast<const uint4*>(kp + 64 * i);  // (a row of 128 bytes by two loads: through the cache)
      const uint8_t* vp = c.v[g] + at + gq * 4 * DH + r * W;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (W == 8) x.v[s][e] = once8(vp + e * DH);
        else x.v[s][e] = make_uint2(__builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(vp + e * DH)), 0u);
      }
    }
  };
  Tile t0;
  float ks = 0.f, vs = 0.f;
  auto scales = [&] {
    ks = id >= 0 ? c.ks[g][(size_t)id * c.HKV + h] : 0.f, vs = id >= 0 ? c.vs[g][(size_t)id * c.HKV + h] : 0.f;
  };
  scales();
  if (t_lo + wave * 32 < t_hi) fetch(t0, t_lo, t_lo + wave * 32);

  uint4 qf[NK];
  float q_scale;
  {
    float x[NK][8];
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const uint4 w = q_raw[k];
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[k][2 * e] = __uint_as_float(v[e] << 16), x[k][2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        most = fmaxf(most, fmaxf(fabsf(x[k][2 * e]), fabsf(x[k][2 * e + 1])));
      }
    }
    most = quarter_max(most);
    const unsigned ex = min(max(__float_as_uint(most) >> 23, 1u), 253u);
    const float f = __uint_as_float((254u - ex) << 23);
    q_scale = __uint_as_float(ex << 23) * (a.scale * LOG2E);
#pragma unroll
    for (int k = 0; k < NK; ++k)
      qf[k] = make_uint4(pack_f16(x[k][0] * f, x[k][1] * f), pack_f16(x[k][2] * f, x[k][3] * f), pack_f16(x[k][4] * f, x[k][5] * f),
                         pack_f16(x[k][6] * f, x[k][7] * f));
  }
  float begin = 0.f;  // of a score's accumulator
  if (KIND == CACHE_INT8) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) sum += sum8(qf[k]);
    begin = quarter_sum(sum) * (-128.f / U_ONE);
    q_scale *= U_ONE;
  }

  f32x4 acc[W];
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = NEG_BIG, l = 0.f, unit = 0.f;  // unit: what the accumulators are to be multiplied by, the largest scale of values so far
  for (int seg = t_lo; seg < t_hi; seg += 64 << pl.page_log2) {
    const int seg_hi = min(t_hi, seg + (64 << pl.page_log2));
    if (seg > t_lo) {
      id = page_of(seg, page_at(seg));
      scales();
      if (seg + wave * 32 < seg_hi) fetch(t0, seg, seg + wave * 32);
    }
    const float unit_now = fmaxf(unit, wave_max(vs));
    if (unit_now > unit) {
      if (seg > t_lo) {
        const float by = other_unit(unit, unit_now, quarter_sum(l), m, l);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] *= by;
      }
      unit = unit_now;
    }
    const float vf = in_units(vs, unit), lv = __builtin_amdgcn_logf(vf), iv = 1.0f / vf;
    auto use = [&](Tile& x, int t) {
      float kf[2], tv[2], ti[2], p[2][4];
      bool ok[2];
      f32x4 z[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int ts = t + 16 * s, pg = (ts - seg) >> pl.page_log2 & 63;
        ok[s] = lane_int(id, pg) >= 0 && ts < seg_hi;
        kf[s] = lane_float(ks, pg) * q_scale, tv[s] = lane_float(lv, pg), ti[s] = lane_float(iv, pg);
        if (KIND == CACHE_E4M3 && (!ok[s] || ts + 16 > seg_hi)) {  // what no token has written may be a NaN
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!ok[s] || ts + 4 * gq + e >= seg_hi) x.v[s][e] = make_uint2(0u, 0u);
        }
        z[s] = f32x4{begin, begin, begin, begin};
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          const uint4& w = x.k[s][k >> 1];
          z[s] = mfma16(k & 1 ? wide8<KIND>(w.z, w.w) : wide8<KIND>(w.x, w.y), qf[k], z[s]);
        }
      }
      float top;
      if (t + 32 > free || !ok[0] || !ok[1]) {  // masked, and scaled here already
        top = NEG_BIG;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int left = ok[s] ? min(sees, seg_hi) - (t + 16 * s) - 4 * gq : 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[s][e] = e < left ? z[s][e] * kf[s] : -__builtin_inff();
            top = fmaxf(top, z[s][e] + tv[s]);
          }
          kf[s] = 1.f;
        }
      } else {
        top = fmaxf(fmaf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), kf[0], tv[0]),
                    fmaf(fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])), kf[1], tv[1]));
      }
      top = quarter_max(top);
      if (__any(top > m)) {
        top = fmaxf(top, m);
        const float keep = fast_exp2(m - top);
        m = top, l *= keep;
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] *= keep;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float off = P_LOG2 - m + tv[s];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[s][e] = fast_exp2(fmaf(z[s][e], kf[s], off));
        l = fmaf((p[s][0] + p[s][1]) + (p[s][2] + p[s][3]), ti[s], l);
      }
      const uint4 pf = make_uint4(pack_f16(p[0][0], p[0][1]), pack_f16(p[0][2], p[0][3]), pack_f16(p[1][0], p[1][1]), pack_f16(p[1][2], p[1][3]));
      if (KIND == CACHE_INT8) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < 4; ++e) x.v[s][e] = make_uint2(turned<KIND>(x.v[s][e].x), W == 8 ? turned<KIND>(x.v[s][e].y) : 0u);
      }
      auto value = [&](auto c_) {
        constexpr int C = decltype(c_)::value, B = C & 3;
        auto word = [&](int s, int e) { return C < 4 ? x.v[s][e].x : x.v[s][e].y; };
        const uint2 a0 = columns2<KIND, B>(word(0, 0), word(0, 1)), a1 = columns2<KIND, B>(word(0, 2), word(0, 3));
        const uint2 a2 = columns2<KIND, B>(word(1, 0), word(1, 1)), a3 = columns2<KIND, B>(word(1, 2), word(1, 3));
        acc[C] = mfma16(make_uint4(a0.x, a1.x, a2.x, a3.x), pf, acc[C]);
        acc[C + 1] = mfma16(make_uint4(a0.y, a1.y, a2.y, a3.y), pf, acc[C + 1]);
      };
      value(std::integral_constant<int, 0>{});
      value(std::integral_constant<int, 2>{});
      if constexpr (W == 8) {
        value(std::integral_constant<int, 4>{});
        value(std::integral_constant<int, 6>{});
      }
    };
    int t = seg + wave * 32;
    Tile t1;  // one tile ahead: what a wave waits for was asked for a tile ago
    constexpr int STEP = NW * 32;
    for (; t < seg_hi; t += 2 * STEP) {
      if (t + STEP < seg_hi) fetch(t1, seg, t + STEP);
      use(t0, t);
      if (t + STEP < seg_hi) {
        if (t + 2 * STEP < seg_hi) fetch(t0, seg, t + 2 * STEP);
        use(t1, t + STEP);
      }
    }
  }
  l = quarter_sum(l) * (1.0f / P_ONE);
  const float one = unit * (KIND == CACHE_INT8 ? U_ONE / P_ONE : 1.0f / P_ONE);

  if (gq == 0) w_ml[wave * 16 + r] = make_float2(m, l);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const f32x4 v = f32x4{acc[i][e], acc[i + 1][e], acc[i + 2][e], acc[i + 3][e]};
      *reinterpret_cast<f32x4*>(w_o + (wave * 16 + r) * (DH + 4) + W * (4 * gq + e) + i) = v * one;
    }
  __syncthreads();
  constexpr int C = W * 4 / NW, PER_ROW = 4 * NW;  // joined by PER_ROW threads a row, C columns each
  const int jr = tid / PER_ROW, at = tid % PER_ROW, d0 = at * C;
  if (first + jr >= rows) return;
  float mm = NEG_BIG;
#pragma unroll
  for (int w = 0; w < NW; ++w) mm = fmaxf(mm, w_ml[w * 16 + jr].x);
  float ll = 0.f, o[C];
#pragma unroll
  for (int i = 0; i < C; ++i) o[i] = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = fast_exp2(w_ml[w * 16 + jr].x - mm);
    ll += w_ml[w * 16 + jr].y * f;
#pragma unroll
    for (int i = 0; i < C; ++i) o[i] += w_o[(w * 16 + jr) * (DH + 4) + d0 + i] * f;
  }
  const int tok = sq.row0 + (first + jr) / share, head = h * share + (first + jr) % share;
  if (pl.n_split == 1) {
    const float f = ll > 0.f ? 1.0f / ll : (ll == 0.f ? 0.f : ll);
    uint32_t* dst = reinterpret_cast<uint32_t*>(a.o[g] + (size_t)tok * a.ld_o + (size_t)head * DH + d0);
#pragma unroll
    for (int i = 0; i < C; i += 2) dst[i >> 1] = pack_bf16(o[i] * f, o[i + 1] * f);
    if (a.lse[g] && at == 0) a.lse[g][(size_t)tok * a.H + head] = ll > 0.f ? mm * LN2 + __logf(ll) : (ll == 0.f ? -__builtin_inff() : ll);
  } else {
    const size_t part = ((size_t)tok * a.H + head) * pl.n_split + split;
    float* po = static_cast<float*>(a.ws[g]) + part * DH + d0;
#pragma unroll
    for (int i = 0; i < C; ++i) po[i] = o[i];
    float2* ml = reinterpret_cast<float2*>(static_cast<float*>(a.ws[g]) + (size_t)c.n_tok * a.H * pl.n_split * DH);
    if (at == 0) ml[part] = make_float2(mm, ll);
  }
}

// ---- many rows of a key/value head ----------------------------------------------------------------------------------------
// NW waves, 32 rows each, share tiles of 64 keys through LDS, as f16 (row-major, 16-byte chunks XOR-ed by the row so that reads of 16 rows at one
// chunk and transposing reads both spread over the banks): codes are widened once for all of a workgroup's rows on their way there.  The
// next tile's codes are in registers while this one's products run; one barrier a tile.  v_mfma_f32_32x32x16_f16:
//   S^T[t,i] = K Q^T (lane: query l%32; accumulator rows 8q + 4(l/32) + e),  O^T[d,i] += V^T P^T, P from the accumulators as they are, V^T by transposing
//   LDS reads.
// A page's scale of the keys is in the factor of its scores, that of the values in the exponent of its weights, as above: neither costs an
// instruction a score.  Weights are rounded to f16 (11 bits, against the 9 that the result keeps) with a factor of 2^7, so that it holds them down to
// 2^-31 of what the row's largest gives.  What a window of 512 pages is (id and scales) waits in LDS, too.
// 8 prompts of up to 2048 tokens, 32 heads of 128, int8, causal: 138 GFLOP of visible pairs in 209 us back to back, 660 TFLOP/s (from an idle chip 240; the
// 16-row tiles above: 638).  Bound by the chain product, maximum, exponential, product of each half tile, which two waves a SIMD do not cover: the vector
// unit works for 53 % of the cycles (exponentials, maxima, widening), the matrix cores for 32 %, both for 13 % of them, neither for 28 %.
typedef __attribute__((ext_vector_type(16))) float f32x16;
__device__ __forceinline__ f32x16 mfma32(const uint4& a, const uint4& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// XOR term of a row's chunks: 16 rows of 256 bytes (128 bytes) need 16 (8) different terms, and 4 rows in a row must move a group of 4 chunks
template <int DH>
__device__ __forceinline__ int swz(int row) {
  return DH == 128 ? 4 * (row & 3) + ((row >> 2) & 3) : 4 * ((row >> 1) & 1) + ((row >> 2) & 3);
}
// Eight keys of one column per lane: rows r and r + 8 .. of the tile, r = row0 + 4(l/32) + {0..3}, by two transposing reads (within 16 lanes, lane j
// supplies four columns of row j/4 and lane i receives column i of rows 0..3)
struct ColumnsAt { unsigned a0, a1; };
template <int DH>
__device__ __forceinline__ ColumnsAt columns_at(unsigned tile, int col0, int lane) {
  constexpr int NCH = DH / 8;
  const int j = lane & 15, grp = lane >> 4, col = col0 + 16 * (grp & 1) + 4 * (j & 3), kc = col >> 3, half = (col >> 2) & 1;
  const int r0 = 4 * (grp >> 1) + (j >> 2), r1 = r0 + 8;
  return {tile + (unsigned)((r0 * NCH + (kc ^ swz<DH>(r0))) * 16 + half * 8), tile + (unsigned)((r1 * NCH + (kc ^ swz<DH>(r1))) * 16 + half * 8)};
}
__device__ __forceinline__ uint4 read_columns(const ColumnsAt& c, unsigned off) {
  typedef __attribute__((ext_vector_type(4))) short s16x4;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(c.a0 + off)));
  const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(c.a1 + off)));
  return make_uint4(lo.x, lo.y, hi.x, hi.y);
}
// What wide8 gives, of int8 without the 128: code 2^-24
template <int KIND>
__device__ __forceinline__ uint4 codes_only(const uint4& v) {
  if (KIND == CACHE_E4M3) return v;
  auto one = [](uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, w) + __builtin_bit_cast(f16x2, 0x80808080u)); };
  return make_uint4(one(v.x), one(v.y), one(v.z), one(v.w));
}
__device__ __forceinline__ void store16(uint4* p, const uint4& v) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  *reinterpret_cast<u32x4*>(p) = u32x4{v.x, v.y, v.z, v.w};
}
constexpr int WINDOW = 512;
template <int DH>
constexpr int prompt_lds() { return 2 * 2 * 64 * DH * 2 + 4 * WINDOW * 4; }

// The sequence of a place in the grid's rows.  Workgroups go to the chip's parts (8 XCDs, 4 shader engines in each) by their number modulo 32, as the
// times show: were the sequence the place itself, a part would have the same sequences over and over, some the long ones.  So where rows of the grid
// fall to the parts alike again, they begin one sequence further (8 prompts of 1024 to 2048 tokens, 32 query heads over 8: 190 us instead of 275, over 1:
// 188, 301).  Single tokens take the same time either way.
__device__ __forceinline__ int sequence_of(int slot, int B) {
  const int alike = max(5 - __builtin_ctz(gridDim.x), 0);  // log2 of the rows until then
  return (int)((unsigned)(slot + (blockIdx.y >> alike) + blockIdx.z) % (unsigned)B);
}

// blockIdx: x sequence and key/value head (the blocks of one head run on one XCD where their number is a multiple of 8), y run of keys and row block, the
// last (longest) row blocks first; z model.  BIG: a tile lies in one page.
template <int KIND, int DH, int NW, bool BIG>
__global__ __launch_bounds__(NW * 64, 2) void cache_prompt_kernel(const CacheAttnArgs a, const CacheAttnPlan pl) {
  constexpr int NT = NW * 64, NCH = DH / 8, NK = DH / 16, NC = DH / 32, BUF = 2 * 64 * NCH;  // chunks of a buffer: K, then V
  constexpr int LOADS = 2 * 64 * (DH / 16) / NT;                                             // of 16 codes per thread and tile
  extern __shared__ __attribute__((aligned(256))) uint4 lds[];
  int* const s_id = reinterpret_cast<int*>(lds + 2 * BUF);
  float* const s_ks = reinterpret_cast<float*>(s_id + WINDOW);
  float* const s_vs = s_ks + WINDOW;  // of values: the scale, then its log2 in units of the largest so far
  float* const s_vi = s_vs + WINDOW;  // 2^ less that
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 31, g = lane >> 5;
  const int gi = blockIdx.z, slot = blockIdx.x / c.HKV, h = blockIdx.x - slot * c.HKV, b = sequence_of(slot, c.B);
  const int split = blockIdx.y / pl.n_rt, blk = pl.n_rt - 1 - (blockIdx.y - split * pl.n_rt);
  const CacheSeq sq = cache_seq(c, b);
  const int share = a.H / c.HKV, rows = sq.n * share, first = blk * NW * 32;
  if (first >= rows) return;
  auto sees_of = [&](int row) { return row < rows ? (a.causal ? max(sq.pos0 + row / share + 1, 0) : sq.len) : 0; };
  const int row = first + wave * 32 + li, sees = sees_of(row), rc = min(row, rows - 1), j = rc / share, hq = h * share + rc - j * share;
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int t_lo = split * pl.chunk, t_hi = uniform(min(t_lo + pl.chunk, sees_of(min(first + NW * 32, rows) - 1)));
  const int wave_last = min(first + wave * 32 + 32, rows) - 1, wave_all = uniform(first + wave * 32 < rows ? min(sees_of(wave_last), t_hi) : 0);
  const int wave_free = uniform(first + wave * 32 + 32 <= rows ? min(sees_of(first + wave * 32), t_hi) : 0);  // keys that all of the wave's rows see

  uint4 qf[NK];
  float q_scale;
  {
    const bf16_t* q = a.q[gi] + (size_t)(sq.row0 + j) * a.ld_q + (size_t)hq * DH + 8 * g;
    uint4 raw[NK];
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) raw[k] = *reinterpret_cast<const uint4*>(q + 16 * k);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const uint32_t v[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(__uint_as_float(v[e] << 16)), fabsf(__uint_as_float(v[e] & 0xffff0000u))));
    }
    const float2 both = wave_swap32(most);
    most = fmaxf(both.x, both.y);
    const unsigned ex = min(max(__float_as_uint(most) >> 23, 1u), 253u);
    const float f = __uint_as_float((254u - ex) << 23);
    q_scale = __uint_as_float(ex << 23) * (a.scale * LOG2E);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      uint32_t v[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = pack_f16(__uint_as_float(v[e] << 16) * f, __uint_as_float(v[e] & 0xffff0000u) * f);
      qf[k] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }

  float begin = 0.f;  // of a score's accumulator
  if (KIND == CACHE_INT8) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) sum += sum8(qf[k]);
    const float2 both = wave_swap32(sum);
    begin = (both.x + both.y) * (-128.f / U_ONE);
    q_scale *= U_ONE;
  }
  const uint4* kr[NK];
  ColumnsAt vc[NC];
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)reinterpret_cast<const char*>(lds);
#pragma unroll
  for (int k = 0; k < NK; ++k) kr[k] = lds + li * NCH + ((2 * k + g) ^ swz<DH>(li));
#pragma unroll
  for (int i = 0; i < NC; ++i) vc[i] = columns_at<DH>(lds0 + 64 * NCH * 16, 32 * i, lane);

  f32x16 acc[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
  float m = NEG_BIG, l = 0.f, unit = 0.f;
  int win = 0;       // the window's first page
  auto window = [&](int key) {
    win = key >> pl.page_log2;
    // as many pages as the tiles ask for, two ahead of the last one
    const int n = uniform((int)min((int64_t)WINDOW, (((int64_t)t_hi - key + 191) >> pl.page_log2) + 1));
    __syncthreads();
    for (int p = tid; p < n; p += NT) {
      int id = -1;
      float ks = 0.f, vs = 0.f;
      if (((int64_t)(win + p) << pl.page_log2) < t_hi) {
        id = c.table[(size_t)b * c.max_pages + win + p];
        if ((unsigned)id >= (unsigned)c.n_pages) id = -1;
        else ks = c.ks[gi][(size_t)id * c.HKV + h], vs = c.vs[gi][(size_t)id * c.HKV + h];
      }
      s_id[p] = id, s_ks[p] = ks, s_vs[p] = vs;
    }
    __syncthreads();
    float most = unit;
    for (int p = lane; p < n; p += 64) most = fmaxf(most, s_vs[p]);
    most = wave_max(most);
    if (most > unit) {
      if (key > t_lo) {
        const float2 both = wave_swap32(l);
        const float by = other_unit(unit, most, both.x + both.y, m, l);
#pragma unroll
        for (int i = 0; i < NC; ++i) acc[i] *= by;
      }
      unit = most;
    }
    __syncthreads();  // every wave has read the scales
    for (int p = tid; p < n; p += NT) {
      const float f = in_units(s_vs[p], unit);
      s_vs[p] = __builtin_amdgcn_logf(f), s_vi[p] = 1.0f / f;
    }
    __syncthreads();
  };
  uint4 raw[LOADS];
  // load i of this thread: 16 codes of a tile's keys or, from KEY_LOADS on, values
  constexpr int CODES = 64 * (DH / 16);
  static_assert(CODES % NT == 0, "a load is one of keys for all threads, or one of values");
  constexpr int KEY_LOADS = CODES / NT;
  // (neighbouring rows of a tile would write to the same banks: rows r and r + 4 are neighbours here)
  auto row_of = [&](int i) {
    const int q = ((i * NT + tid) & (CODES - 1)) / (DH / 16);
    return (q & ~7) | (q & 1) << 2 | (q >> 1 & 3);
  };
  auto col_of = [&](int i) { return tid & (DH / 16 - 1); };
  // What the scalar unit knows of a tile: its pages (of 16 keys each, or the one).  Asked for a tile ahead, like the codes.
  constexpr int NG = BIG ? 1 : 4;
  struct Pages { int id[NG]; float ks[NG], lv[NG], iv[NG]; };
  auto pages_at = [&](int t) {
    Pages p;
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      const int at = min(((t + 16 * x) >> pl.page_log2) - win, WINDOW - 1);
      p.id[x] = s_id[at], p.ks[x] = s_ks[at], p.lv[x] = s_vs[at], p.iv[x] = s_vi[at];
    }
    return p;
  };
  auto settle = [&](const Pages& v) {
    Pages p;
    auto one = [](float f) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(f))); };
#pragma unroll
    for (int x = 0; x < NG; ++x) p.id[x] = __builtin_amdgcn_readfirstlane(v.id[x]), p.ks[x] = one(v.ks[x]), p.lv[x] = one(v.lv[x]), p.iv[x] = one(v.iv[x]);
    return p;
  };
  auto fetch = [&](int t, const Pages& pg) {
    if constexpr (BIG) {
      const int id = pg.id[0];
      const size_t at = (size_t)max(id, 0) * c.page_bytes + ((size_t)h * c.page + (t & (c.page - 1))) * DH;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) raw[i] = *reinterpret_cast<const uint4*>((i < KEY_LOADS ? c.k[gi] : c.v[gi]) + at + (unsigned)(row_of(i) * DH + col_of(i) * 16));
      if (KIND == CACHE_E4M3 && (id < 0 || t + 64 > t_hi)) {  // what no token has written may be a NaN
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          if (id < 0 || t + row_of(i) >= t_hi) raw[i] = make_uint4(0, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int key = t + row_of(i), pid = key < t_hi ? s_id[(key >> pl.page_log2) - win] : -1;
        const uint8_t* p = (i < KEY_LOADS ? c.k[gi] : c.v[gi]) + (size_t)max(pid, 0) * c.page_bytes + ((size_t)h * c.page + (key & (c.page - 1))) * DH + col_of(i) * 16;
        raw[i] = pid >= 0 ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
      }
    }
  };
  auto put = [&](uint4* tile) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = row_of(i), kc = 2 * col_of(i);
      uint4 lo = wide8<KIND>(raw[i].x, raw[i].y), hi = wide8<KIND>(raw[i].z, raw[i].w);
      uint4* p = tile + r * NCH;
      if (i >= KEY_LOADS) lo = codes_only<KIND>(lo), hi = codes_only<KIND>(hi), p += 64 * NCH;
      store16(p + (kc ^ swz<DH>(r)), lo);
      store16(p + ((kc + 1) ^ swz<DH>(r)), hi);
    }
  };

  Pages now{}, next{};
  int w_hi = 0;  // the end of the window's keys
  auto tile = [&](auto buf_, int t) {
    constexpr int B = decltype(buf_)::value * BUF;
    const bool more = t + 64 < w_hi;
    if (more) fetch(t + 64, next);
    unsigned gone = 0;  // 16-key groups that are not there
#pragma unroll
    for (int x = 0; x < NG; ++x) gone |= now.id[x] < 0 ? (BIG ? 15u : 1u << x) : 0u;
    if (t < wave_all) {
      // 32 keys at a time, so that the products of one half stand beside the exponentials of the other
      const bool edge = t + 64 > wave_free || gone;
      f32x16 s;
      uint4 kf[NK];
      auto keys = [&](int sub) {  // all fragments asked for at once (left alone, each read is waited for where it stands)
#pragma unroll
        for (int k = 0; k < NK; ++k) kf[k] = kr[k][B + sub * 32 * NCH];
        __builtin_amdgcn_sched_barrier(0);
      };
      auto scores = [&] {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int k = 0; k < NK; ++k) s = mfma32(kf[k], qf[k], s);
      };
      float f[2], start = begin;
      auto highest = [&](int sub) {  // and the masks; masked scores are scaled at once
        float top = NEG_BIG;
        f[0] = now.ks[2 * sub % NG] * q_scale, f[1] = now.ks[(2 * sub + 1) % NG] * q_scale;
        if (edge) {
          const int left = min(sees, t_hi) - t - 4 * g;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int here = gone >> (2 * sub + x) & 1 ? 0 : left;
            float most = -__builtin_inff();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float z = 16 * (2 * sub + x) + 8 * (e >> 2) + (e & 3) < here ? (s[8 * x + e] + begin) * f[x] : -__builtin_inff();
              s[8 * x + e] = z;
              most = fmaxf(most, z);
            }
            top = fmaxf(top, most + now.lv[(2 * sub + x) % NG]);
            f[x] = 1.f;
          }
          start = 0.f;
        } else {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float most = s[8 * x];
#pragma unroll
            for (int e = 1; e < 8; ++e) most = fmaxf(most, s[8 * x + e]);
            top = fmaxf(top, fmaf(most + start, f[x], now.lv[(2 * sub + x) % NG]));
          }
        }
        const float2 both = wave_swap32(top);
        top = fmaxf(both.x, both.y);
        // weights are 2^7 of those by the maximum that is held: it may lag by 2^8 (their f16 ends at 2^16) before accumulators are scaled again
        if (__any(top > m + 8.f)) {
          top = fmaxf(top, m);
          const float keep = fast_exp2(m - top);
          l *= keep;
#pragma unroll
          for (int i = 0; i < NC; ++i) acc[i] *= keep;
          m = top;
        }
      };
      uint4 pf[2];
      auto weights = [&](int sub) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float p[8];
          const float off = fmaf(start, f[x], 7.f - m + now.lv[(2 * sub + x) % NG]);
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = fast_exp2(fmaf(s[8 * x + e], f[x], off));
          l += (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]))) * now.iv[(2 * sub + x) % NG];
          pf[x] = make_uint4(pack_f16(p[0], p[1]), pack_f16(p[2], p[3]), pack_f16(p[4], p[5]), pack_f16(p[6], p[7]));
        }
      };
      auto results = [&](int sub) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < NC; ++i) acc[i] = mfma32(read_columns(vc[i], (unsigned)((B + (2 * sub + x) * 16 * NCH) * 16)), pf[x], acc[i]);
      };
      keys(0);
      scores();
      keys(1);
      highest(0);
      weights(0);
      scores();
      results(0);
      highest(1);
      weights(1);
      results(1);
    }
    const Pages then = pages_at(t + 128);
    if (more) put(lds + (BUF - B));
    now = next, next = settle(then);
    __syncthreads();
  };
  for (int w = t_lo; w < t_hi; w = w_hi) {
    w_hi = uniform((int)min((int64_t)t_hi, (int64_t)w + ((int64_t)WINDOW << pl.page_log2)));
    window(w);
    now = settle(pages_at(w)), next = settle(pages_at(w + 64));
    fetch(w, now);
    put(lds);
    __syncthreads();
    for (int t = w; t < w_hi; t += 128) {
      tile(std::integral_constant<int, 0>{}, t);
      if (t + 64 < w_hi) tile(std::integral_constant<int, 1>{}, t + 64);
    }
  }

  const float2 both = wave_swap32(l);
  l = (both.x + both.y) * (1.0f / 128.f);
  if (row >= rows) return;
  const float one = unit * (KIND == CACHE_INT8 ? U_ONE / 128.f : 1.0f / 128.f);
  const int tok = sq.row0 + j;
  if (pl.n_split == 1) {
    const float f = l > 0.f ? one / l : (l == 0.f ? 0.f : l);
    bf16_t* dst = a.o[gi] + (size_t)tok * a.ld_o + (size_t)hq * DH;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<uint2*>(dst + 32 * i + 8 * q + 4 * g) =
            make_uint2(pack_bf16(acc[i][4 * q] * f, acc[i][4 * q + 1] * f), pack_bf16(acc[i][4 * q + 2] * f, acc[i][4 * q + 3] * f));
    if (a.lse[gi] && !g) a.lse[gi][(size_t)tok * a.H + hq] = l > 0.f ? m * LN2 + __logf(l) : (l == 0.f ? -__builtin_inff() : l);
  } else {
    const size_t part = ((size_t)tok * a.H + hq) * pl.n_split + split;
    float* po = static_cast<float*>(a.ws[gi]) + part * DH;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(po + 32 * i + 8 * q + 4 * g) =
            make_float4(acc[i][4 * q] * one, acc[i][4 * q + 1] * one, acc[i][4 * q + 2] * one, acc[i][4 * q + 3] * one);
    float2* ml = reinterpret_cast<float2*>(static_cast<float*>(a.ws[gi]) + (size_t)c.n_tok * a.H * pl.n_split * DH);
    if (!g) ml[part] = make_float2(m, l);
  }
}

// Whether some sequence of the call has row `tok`, as cache_seq says it (a wave's 64 lanes look at 64 places of q_ptr at a time; the last sequence that
// begins at or before the row is the one that can).
__device__ __forceinline__ bool row_of_call(const CacheArgs& c, int tok, int lane) {
  if (!c.q_ptr) return true;
  int lo = 0, hi = c.B;
  while (true) {
    const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
    const int before = __popcll(__ballot(at < hi && c.q_ptr[min(at, hi - 1)] <= tok));
    if (!before) return false;
    lo += (before - 1) * step, hi = min(lo + step, hi);
    if (step == 1) break;
  }
  const CacheSeq sq = cache_seq(c, lo);
  return tok >= sq.row0 && tok - sq.row0 < sq.n;
}
// The runs' partial sums of one row and head, in ascending order: one wave each.  A lane has the maximum and sum of one run (64 at a time).  Rows of
// no sequence (past q_ptr[B], or past the max_q rows that one may have) have no partial sums and are left alone.
template <int DH>
__global__ __launch_bounds__(64) void cache_attn_join_kernel(const CacheAttnArgs a, const CacheAttnPlan pl) {
  constexpr int E = DH / 64;
  const int g = blockIdx.y, lane = threadIdx.x;
  const int64_t n = (int64_t)a.c.n_tok * a.H, i = blockIdx.x;
  const int tok = (int)(i / a.H), head = (int)(i - (int64_t)tok * a.H);
  const float* po = static_cast<const float*>(a.ws[g]) + (size_t)i * pl.n_split * DH + lane * E;
  const float2* ml = reinterpret_cast<const float2*>(static_cast<const float*>(a.ws[g]) + (size_t)n * pl.n_split * DH) + (size_t)i * pl.n_split;
  if (!row_of_call(a.c, tok, lane)) return;
  float mm = NEG_BIG;
  for (int s0 = 0; s0 < pl.n_split; s0 += 64) mm = fmaxf(mm, s0 + lane < pl.n_split ? ml[s0 + lane].x : NEG_BIG);
  mm = wave_max(mm);
  float ll = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int s0 = 0; s0 < pl.n_split; s0 += 64) {
    const float2 v = s0 + lane < pl.n_split ? ml[s0 + lane] : make_float2(NEG_BIG, 0.f);
    const float w = fast_exp2(v.x - mm);
    ll += wave_sum(v.y * w);
    const int cnt = min(64, pl.n_split - s0);
    for (int s = 0; s < cnt; s += 8) {  // eight loads under way together; past the last run that one again, by 0
      float x[8][E];
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int e = 0; e < E; ++e) x[q][e] = po[(size_t)(s0 + min(s + q, cnt - 1)) * DH + e];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float f = s + q < cnt ? lane_float(w, s + q) : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += x[q][e] * f;
      }
    }
  }
  const float f = ll > 0.f ? 1.0f / ll : (ll == 0.f ? 0.f : ll);
  bf16_t* dst = a.o[g] + (size_t)tok * a.ld_o + (size_t)head * DH + lane * E;
  if (E == 2) *reinterpret_cast<uint32_t*>(dst) = pack_bf16(o[0] * f, o[E - 1] * f);
  else *dst = (bf16_t)pack_bf16(o[0] * f, 0.f);
  if (a.lse[g] && lane == 0) a.lse[g][i] = ll > 0.f ? mm * LN2 + __logf(ll) : (ll == 0.f ? -__builtin_inff() : ll);
}

int floor_log2(int v) { return 31 - __builtin_clz((unsigned)v); }

// Which kernel, with how many waves, and how many runs a sequence's keys are split into; from the host's bounds alone.  All figures in us, heads of 128,
// int8, as (this choice | the other one).
// Prompt kernel or 16-row tiles, by rows of a key/value head.  Up to 64 rows four 16-row tiles read no more than the caches give again (64 rows:
// 13 | 21 for one sequence, 32 | 38 for 8 of 4096 tokens, 63 | 65 for 32); beyond, where the chip is full, one pass over the codes wins (96 rows: 40 |
// 53 and 72 | 93, 256 rows: 71 | 114 and 100 | 201).  Tiles that are few against the keys stay with the 16-row kernel, which has more workgroups (32 heads of one
// sequence of 512 tokens: 16 to 21 | 21 to 27, 16 heads of 700: 20 | 25; but 1352 of four sequences, 2 heads, 1813 keys: 35 | 38, 12 heads of 64
// short prompts: 13 | 31, 96 rows over 32768 keys: 46 | 64).
// Eight waves or four.  Up to 512 tiles, two for a CU, the eight are what keeps loads under way (8 sequences of 32768 tokens, 8 heads: 73 | 78; 32
// of 4096: 42 | 46; 40 to 60 of 4096: 61..73 | 64..82); above, four join faster (72 of 4096: 93 with eight, 98 with four in one run, but 1024 tokens: 21 | 23).
// Runs.  Few tiles: as many as fill the 256 CUs once, of 256 keys at least; where the heads do that already, one, until it is longer than 8192 keys.  Up
// to 640 keys the second launch costs more than it saves (300 tokens: 9 | 11, 513: 9.8 | 11.3; 800: 11.6 in one, 10.9 split).  The prompt kernel's blocks
// run two to a CU: 512 of them, of 256 keys at least (35 and 56 | 53 and 87 with 256 blocks of 512); where
// they fill the CUs once as it is, of 1024 at least (288 blocks: 300 keys 13 | 25 split, 1100 keys 39 | 48, but 4000 keys 102 split, 122 not).
// Rows of a prompt block, heads of 128.  Eight waves widen a tile for 256 rows, not 128, but have a CU to themselves, and where the keys are those of the rows
// a block's first waves wait for its last.  Worth it for few rows behind many keys (512 tokens behind 30000, four heads sharing: 260 | 283, behind
// 7000, none sharing: 84 | 90), level for 4 times the keys (227 | 228), not for whole prompts (8 of 2048, four heads sharing: 275 | 292).
CacheAttnPlan plan_of(const CacheArgs& c, int H) {
  CacheAttnPlan p{};
  p.page_log2 = floor_log2(c.page);
  const int64_t rows = (int64_t)c.max_q * (H / c.HKV), len = c.max_len;
  const int64_t heads = (int64_t)c.G * c.B * c.HKV, tiles = heads * ((rows + 15) / 16);
  p.prompt = rows > 64 && (tiles > 1024 || tiles * len > 640 * 1024);
  if (p.prompt) p.waves = c.DH == 128 && rows >= 256 && len >= 8 * (int64_t)c.max_q ? 8 : 4;
  else p.waves = tiles <= 512 ? 8 : 4;
  const int64_t per = p.prompt ? p.waves * 32 : 16;
  p.n_rt = (int)((rows + per - 1) / per);
  const int64_t base = heads * p.n_rt;
  int64_t n;
  if (p.prompt) {
    const int64_t blocks = p.waves == 8 ? 256 : 512;
    n = base > blocks / 2 ? std::max(std::min((blocks + base - 1) / base, len / 1024), (int64_t)1) : std::min((blocks + base - 1) / base, (len + 255) / 256);
  } else {
    n = len <= 640 ? 1 : std::min(std::max(256 / base, (len + 8191) / 8192), (len + 255) / 256);
  }
  p.chunk = (int)(((len + n - 1) / n + 127) / 128 * 128);
  p.n_split = (int)((len + p.chunk - 1) / p.chunk);
  return p;
}

template <int KIND, int DH>
hipError_t run_attn(const CacheAttnArgs& a, const CacheAttnPlan& p, dim3 grid, hipStream_t s) {
  if (p.prompt) {
    const bool big = p.page_log2 >= 6;
    if constexpr (DH == 128) {
      if (p.waves == 8) {
        if (big) hipLaunchKernelGGL((cache_prompt_kernel<KIND, DH, 8, true>), grid, dim3(512), prompt_lds<DH>(), s, a, p);
        else hipLaunchKernelGGL((cache_prompt_kernel<KIND, DH, 8, false>), grid, dim3(512), prompt_lds<DH>(), s, a, p);
        return hipGetLastError();
      }
    }
    if (big) hipLaunchKernelGGL((cache_prompt_kernel<KIND, DH, 4, true>), grid, dim3(256), prompt_lds<DH>(), s, a, p);
    else hipLaunchKernelGGL((cache_prompt_kernel<KIND, DH, 4, false>), grid, dim3(256), prompt_lds<DH>(), s, a, p);
  }
  else if (p.waves == 4) hipLaunchKernelGGL((cache_attn_kernel<KIND, DH, 4>), grid, dim3(256), (attn_lds<DH, 4>()), s, a, p);
  else hipLaunchKernelGGL((cache_attn_kernel<KIND, DH, 8>), grid, dim3(512), (attn_lds<DH, 8>()), s, a, p);
  return hipGetLastError();
}
template <int KIND, int DH>
hipError_t attn_init_kind() {
  hipError_t e = hipFuncSetAttribute((const void*)cache_attn_kernel<KIND, DH, 8>, hipFuncAttributeMaxDynamicSharedMemorySize, attn_lds<DH, 8>());
  if (e != hipSuccess) return e;
  if constexpr (DH == 128) {
    e = hipFuncSetAttribute((const void*)cache_prompt_kernel<KIND, DH, 8, false>, hipFuncAttributeMaxDynamicSharedMemorySize, prompt_lds<DH>());
    if (e != hipSuccess) return e;
    e = hipFuncSetAttribute((const void*)cache_prompt_kernel<KIND, DH, 8, true>, hipFuncAttributeMaxDynamicSharedMemorySize, prompt_lds<DH>());
    if (e != hipSuccess) return e;
  }
  e = hipFuncSetAttribute((const void*)cache_prompt_kernel<KIND, DH, 4, false>, hipFuncAttributeMaxDynamicSharedMemorySize, prompt_lds<DH>());
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)cache_prompt_kernel<KIND, DH, 4, true>, hipFuncAttributeMaxDynamicSharedMemorySize, prompt_lds<DH>());
}

}  // namespace

size_t cache_attn_ws_bytes(const CacheArgs& c, int H) {
  const CacheAttnPlan p = plan_of(c, H);
  // (whole 16 bytes, so that scratch of several models lies in one allocation, each on its alignment)
  return p.n_split == 1 ? 0 : ((size_t)c.n_tok * H * p.n_split * (c.DH + 2) * sizeof(float) + 15) / 16 * 16;
}

void cache_attn_plan(const CacheArgs& c, int H, int32_t plan[3]) {
  const CacheAttnPlan p = plan_of(c, H);
  plan[0] = p.prompt ? p.waves * 32 : 16, plan[1] = p.waves, plan[2] = p.n_split;
}

const char* cache_attn_sizes_refusal(const CacheArgs& c, int H) {
  if (const char* why = cache_sizes_refusal(c)) return why;
  if (H < 1 || H % c.HKV) return "H is no multiple of HKV";
  if ((int64_t)c.max_q * (H / c.HKV) > 0x7fffffffLL - 1024) return "too many rows of one key/value head";
  return nullptr;
}

const char* cache_attn_refusal(const CacheAttnArgs& a) {
  if (const char* why = cache_refusal(a.c)) return why;
  const CacheArgs& c = a.c;
  if (const char* why = cache_attn_sizes_refusal(c, a.H)) return why;
  if (a.ld_q % 8 || a.ld_o % 8 || (int64_t)a.ld_q < (int64_t)a.H * c.DH || (int64_t)a.ld_o < (int64_t)a.H * c.DH)
    return "ld_q or ld_o is less than a row or no multiple of 8";
  if (!(a.scale > 0.f) || a.scale > 1e30f) return "scale is positive and finite";
  for (int g = 0; g < c.G; ++g) {
    if (!a.q[g] || !a.o[g] || ((uintptr_t)a.q[g] | (uintptr_t)a.o[g]) % 16) return "q or o is NULL or not 16-byte aligned";
    if ((a.lse[g] != nullptr) != (a.lse[0] != nullptr)) return "lse for all models or for none";
    if ((a.ws[g] != nullptr) != (a.ws[0] != nullptr) || (uintptr_t)a.ws[g] % 16) return "ws for all models or for none, 16-byte aligned";
  }
  return nullptr;
}

hipError_t cache_attn_init() {
  hipError_t e;
  if ((e = attn_init_kind<CACHE_INT8, 64>()) != hipSuccess) return e;
  if ((e = attn_init_kind<CACHE_INT8, 128>()) != hipSuccess) return e;
  if ((e = attn_init_kind<CACHE_E4M3, 64>()) != hipSuccess) return e;
  return attn_init_kind<CACHE_E4M3, 128>();
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t s) {
  const CacheArgs& c = a.c;
  CacheAttnPlan p = plan_of(c, a.H);
  if (p.n_split > 1 && (!a.ws[0] || a.ws_bytes < cache_attn_ws_bytes(c, a.H))) p.n_split = 1, p.chunk = (c.max_len + 127) / 128 * 128;
  const int64_t bh = (int64_t)c.B * c.HKV, sr = (int64_t)p.n_split * p.n_rt;
  if (bh > 0x7fffffffLL || sr > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)bh, (unsigned)sr, c.G);
  hipError_t e;
  if (c.kind == CACHE_INT8) e = c.DH == 64 ? run_attn<CACHE_INT8, 64>(a, p, grid, s) : run_attn<CACHE_INT8, 128>(a, p, grid, s);
  else e = c.DH == 64 ? run_attn<CACHE_E4M3, 64>(a, p, grid, s) : run_attn<CACHE_E4M3, 128>(a, p, grid, s);
  if (e != hipSuccess) return e;
  if (p.n_split == 1) return hipSuccess;
  if ((int64_t)c.n_tok * a.H > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 join((unsigned)((int64_t)c.n_tok * a.H), c.G);
  if (c.DH == 64) hipLaunchKernelGGL((cache_attn_join_kernel<64>), join, dim3(64), 0, s, a, p);
  else hipLaunchKernelGGL((cache_attn_join_kernel<128>), join, dim3(64), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace hydra
