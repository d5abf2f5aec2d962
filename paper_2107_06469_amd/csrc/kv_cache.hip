// Keys and values of new tokens into a paged cache of 8-bit codes, with the position rotation of queries and keys on the way.
//   rotation (x: a head's first r = rot_dim columns, c and s: cosine and sine of the token's position):
//     halves:     x'[i] = x[i] c[i] - x[i + r/2] s[i],  x'[i + r/2] = x[i + r/2] c[i] + x[i] s[i],  i < r/2;  neighbours: the same with 2i, 2i + 1
//   a page (of one head): s = max(s_before, max |x'| / Q, 2^-126), Q = 127 (int8) or 448 (e4m3), s_before = 0 where slot 0 is new;
//     where s grew, the codes held become round(code * (s_before / s));  new codes are round(x' * (1 / s)), to nearest even.
// Every product and sum of a value is rounded by itself (no contraction), so a code depends on nothing but the formula.
// One workgroup has one page of one head of keys or values, or a run of query rows: new rows pass through registers once (maximum, then codes),
// and no two workgroups touch one scale.  Bound by HBM for whole prompts (eight of up to 2048 tokens, 32 heads of 128, e4m3: 463 MB in 106 us,
// 4.4 TB/s where a copy reaches 5.1; 397 us when the rows were read once for the maximum and again for the codes), by the launch and three
// dependent loads (length, page, scale) for single tokens (3.6 us for one sequence and for 2 x 64).
#include <float.h>

#include "kernels.h"
#include "wave_math.h"

namespace hydra {
namespace {

constexpr float LEAST_SCALE = 1.17549435e-38f;  // 2^-126: its reciprocal is finite

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// four codes in one word: x * f to nearest even, at most the largest code; NaN becomes 0
template <int KIND>
__device__ __forceinline__ uint32_t to_codes(float x0, float x1, float x2, float x3, float f) {
#pragma clang fp contract(off)
  constexpr float TOP = KIND == CACHE_INT8 ? 127.f : 448.f;
  const float x[4] = {x0, x1, x2, x3};
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float v = x[i] * f;
    y[i] = v == v ? fminf(fmaxf(v, -TOP), TOP) : 0.f;
  }
  if (KIND == CACHE_INT8) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)rintf(y[i]) & 0xffu) << (8 * i);
    return w;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}
// four codes by another scale
template <int KIND>
__device__ __forceinline__ uint32_t again(uint32_t w, float f) {
  if (KIND == CACHE_INT8)
    return to_codes<KIND>((float)((int)(w << 24) >> 24), (float)((int)(w << 16) >> 24), (float)((int)(w << 8) >> 24), (float)((int)w >> 24), f);
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return to_codes<KIND>(a.x, a.y, b.x, b.y, f);
}

// Sixteen values of a row in registers: two runs of 8 columns.
struct Unit {
  float x[16];
  __device__ __forceinline__ void load(const bf16_t* row, int2 at) {
    const uint4 a = *reinterpret_cast<const uint4*>(row + at.x), b = *reinterpret_cast<const uint4*>(row + at.y);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[2 * i] = bf_lo(w[i]), x[2 * i + 1] = bf_hi(w[i]);
  }
};

// Unit u of a head's row: the two runs of 8 columns that a rotation by halves turns into one another (columns past rot_dim go by in order).
__device__ __forceinline__ int2 unit_columns(int u, int rot_dim) {
  const int turned = rot_dim >> 4;
  return u < turned ? make_int2(8 * u, 8 * u + (rot_dim >> 1)) : make_int2(16 * u, 16 * u + 8);
}
// cs: the position's row of the table.  Of the two kinds of pairs one is this launch's; columns past rot_dim have none.
template <int ROT>
__device__ __forceinline__ void rotate(Unit& u, int2 at, int rot_dim, const float* cs) {
#pragma clang fp contract(off)
  if (ROT == ROT_NONE || at.x >= rot_dim) return;
  const float* sn = cs + (rot_dim >> 1);
  float c[8], s[8];
  const int ca = ROT == ROT_HALVES ? at.x : at.x >> 1, cb = ROT == ROT_HALVES ? at.x + 4 : at.y >> 1;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float4 cv = *reinterpret_cast<const float4*>(cs + (h ? cb : ca)), sv = *reinterpret_cast<const float4*>(sn + (h ? cb : ca));
    c[4 * h] = cv.x, c[4 * h + 1] = cv.y, c[4 * h + 2] = cv.z, c[4 * h + 3] = cv.w;
    s[4 * h] = sv.x, s[4 * h + 1] = sv.y, s[4 * h + 2] = sv.z, s[4 * h + 3] = sv.w;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float &a = u.x[ROT == ROT_HALVES ? i : 2 * i], &b = u.x[ROT == ROT_HALVES ? 8 + i : 2 * i + 1];
    const float ac = a * c[i], bs = b * s[i], bc = b * c[i], as = a * s[i];
    a = ac - bs;
    b = bc + as;
  }
}

// NT threads; a page's new rows are at most NT * UPT units.  blockIdx: x the pages and heads of keys and values, then the runs of query rows;
// y the sequence; z the model.
template <int KIND, int ROT, int NT, int UPT>
__global__ __launch_bounds__(NT) void append_kernel(const AppendArgs a) {
  const CacheArgs& c = a.c;
  const int g = blockIdx.z, b = blockIdx.y, tid = threadIdx.x;
  const int upr_log2 = c.DH == 128 ? 3 : 2, upr = 1 << upr_log2;  // units per head's row
  const CacheSeq s = cache_seq(c, b);
  const bf16_t* const qkv = a.qkv[g] + (size_t)s.row0 * a.ld_qkv;
  int x = blockIdx.x;
  if (x >= a.cache_blocks) {  // query rows
    x -= a.cache_blocks;
    const int u = x * NT + tid, per_row = a.H * upr, j = u / per_row;
    if (j >= s.n || s.pos0 + j < 0) return;
    const int v = u - j * per_row, h = v >> upr_log2;
    const int2 at = unit_columns(v - h * upr, a.rot_dim);
    Unit w;
    w.load(qkv + (size_t)j * a.ld_qkv + h * c.DH, at);
    rotate<ROT>(w, at, a.rot_dim, a.cs + (size_t)(s.pos0 + j) * a.rot_dim);
    bf16_t* dst = a.q[g] + (size_t)(s.row0 + j) * a.ld_q + h * c.DH;
    *reinterpret_cast<uint4*>(dst + at.x) = make_uint4(pack2(w.x[0], w.x[1]), pack2(w.x[2], w.x[3]), pack2(w.x[4], w.x[5]), pack2(w.x[6], w.x[7]));
    *reinterpret_cast<uint4*>(dst + at.y) = make_uint4(pack2(w.x[8], w.x[9]), pack2(w.x[10], w.x[11]), pack2(w.x[12], w.x[13]), pack2(w.x[14], w.x[15]));
    return;
  }
  const int per_page = 2 * c.HKV, nth = x / per_page, hv = x - nth * per_page, h = hv >> 1, is_v = hv & 1;
  const int begin = max(s.pos0, 0), pg = begin / c.page + nth, page0 = pg * c.page;
  const int lo = max(page0, begin), hi = min(page0 + c.page, s.len);
  if (lo >= hi || pg >= c.max_pages) return;
  const unsigned id = (unsigned)c.table[(size_t)b * c.max_pages + pg];
  if (id >= (unsigned)c.n_pages) return;
  float* const scale = (is_v ? c.vs[g] : c.ks[g]) + (size_t)id * c.HKV + h;
  uint8_t* const codes = (is_v ? c.v[g] : c.k[g]) + (size_t)id * c.page_bytes + (size_t)h * c.page * c.DH;
  const bool fresh = lo == page0;
  const float before = fresh ? 0.f : *scale;
  const bf16_t* const src = qkv + (size_t)(a.H + (is_v ? c.HKV : 0) + h) * c.DH;
  const int units = (hi - lo) * upr;
  Unit w[UPT];
#pragma unroll
  for (int i = 0; i < UPT; ++i) {  // every load before the first use; a row past the last one is that one again
    const int u = min(i * NT + tid, units - 1), r = u >> upr_log2;
    w[i].load(src + (size_t)(lo + r - s.pos0) * a.ld_qkv, unit_columns(u - r * upr, a.rot_dim));
  }
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < UPT; ++i) {
    const int u = min(i * NT + tid, units - 1), r = u >> upr_log2;
    if (!is_v) rotate<ROT>(w[i], unit_columns(u - r * upr, a.rot_dim), a.rot_dim, a.cs + (size_t)(lo + r) * a.rot_dim);
#pragma unroll
    for (int e = 0; e < 16; ++e) most = fmaxf(most, fabsf(w[i].x[e]) <= FLT_MAX ? fabsf(w[i].x[e]) : 0.f);
  }
  most = wave_max(most);
  if (NT > 64) {
    __shared__ float part[NT / 64];
    if ((tid & 63) == 0) part[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) most = fmaxf(most, part[i]);
  }
  constexpr float PER_TOP = KIND == CACHE_INT8 ? 1.0f / 127.0f : 1.0f / 448.0f;
  const float now = fmaxf(before, fmaxf(most * PER_TOP, LEAST_SCALE));
  if (!fresh && now > before) {  // what the page holds, by the new scale
    const float f = before / now;
    uint4* p = reinterpret_cast<uint4*>(codes);
    for (int i = tid; i < (lo - page0) * c.DH / 16; i += NT) {
      const uint4 old = p[i];
      p[i] = make_uint4(again<KIND>(old.x, f), again<KIND>(old.y, f), again<KIND>(old.z, f), again<KIND>(old.w, f));
    }
  }
  const float by = 1.0f / now;
#pragma unroll
  for (int i = 0; i < UPT; ++i) {
    const int u = i * NT + tid;
    if (u < units) {
      const int r = u >> upr_log2;
      const int2 at = unit_columns(u - r * upr, a.rot_dim);
      uint8_t* row = codes + (size_t)(lo - page0 + r) * c.DH;
      const float* x = w[i].x;
      *reinterpret_cast<uint2*>(row + at.x) = make_uint2(to_codes<KIND>(x[0], x[1], x[2], x[3], by), to_codes<KIND>(x[4], x[5], x[6], x[7], by));
      *reinterpret_cast<uint2*>(row + at.y) = make_uint2(to_codes<KIND>(x[8], x[9], x[10], x[11], by), to_codes<KIND>(x[12], x[13], x[14], x[15], by));
    }
  }
  if (tid == 0) *scale = now;
}

template <int KIND, int ROT>
void run_append(const AppendArgs& a, dim3 grid, int nt, int upt, hipStream_t s) {
  if (nt == 64) hipLaunchKernelGGL((append_kernel<KIND, ROT, 64, 1>), grid, dim3(64), 0, s, a);
  else if (nt == 128) hipLaunchKernelGGL((append_kernel<KIND, ROT, 128, 1>), grid, dim3(128), 0, s, a);
  else if (upt == 1) hipLaunchKernelGGL((append_kernel<KIND, ROT, 256, 1>), grid, dim3(256), 0, s, a);
  else if (upt == 2) hipLaunchKernelGGL((append_kernel<KIND, ROT, 256, 2>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((append_kernel<KIND, ROT, 256, 4>), grid, dim3(256), 0, s, a);
}
template <int KIND>
void run_append(const AppendArgs& a, dim3 grid, int nt, int upt, hipStream_t s) {
  if (a.rot == ROT_HALVES) run_append<KIND, ROT_HALVES>(a, grid, nt, upt, s);
  else if (a.rot == ROT_NEIGHBOURS) run_append<KIND, ROT_NEIGHBOURS>(a, grid, nt, upt, s);
  else run_append<KIND, ROT_NONE>(a, grid, nt, upt, s);
}

}  // namespace

const char* cache_sizes_refusal(const CacheArgs& c) {
  if (c.kind != CACHE_INT8 && c.kind != CACHE_E4M3) return "kind is neither int8 nor e4m3";
  if (c.DH != 64 && c.DH != 128) return "head width is neither 64 nor 128";
  if (c.page != 16 && c.page != 32 && c.page != 64 && c.page != 128) return "a page has 16, 32, 64 or 128 tokens";
  if (c.B < 1 || c.B > 65535 || c.HKV < 1 || c.HKV > 1024 || c.n_pages < 1 || c.max_pages < 1) return "a count is out of range";
  if (c.max_q < 1 || c.n_tok < 1 || c.max_len < 1) return "max_q, n_tok and max_len are at least 1";
  if ((int64_t)c.max_len > (int64_t)c.max_pages * c.page || c.max_len > (1 << 30)) return "max_len goes past the page table";
  if (c.max_q > c.n_tok) return "max_q is more than n_tok";
  if (c.page_bytes < (size_t)c.HKV * c.page * c.DH || c.page_bytes % 16) return "page_bytes is less than a page or no multiple of 16";
  return nullptr;
}

const char* cache_refusal(const CacheArgs& c) {
  if (const char* why = cache_sizes_refusal(c)) return why;
  if (!c.q_ptr && (c.max_q != 1 || c.n_tok != c.B)) return "without q_ptr every sequence has one token";
  if (!c.table || !c.lens) return "page_table or lens is NULL";
  for (int g = 0; g < c.G; ++g) {
    if (!c.k[g] || !c.v[g] || !c.ks[g] || !c.vs[g]) return "NULL entry";
    if (((uintptr_t)c.k[g] | (uintptr_t)c.v[g]) % 16) return "k and v are 16-byte aligned";
  }
  return nullptr;
}

const char* append_refusal(const AppendArgs& a) {
  if (const char* why = cache_refusal(a.c)) return why;
  const CacheArgs& c = a.c;
  if (a.H < 1 || a.H % c.HKV) return "H is no multiple of HKV";
  if (a.ld_qkv % 8 || (int64_t)a.ld_qkv < ((int64_t)a.H + 2 * c.HKV) * c.DH) return "ld_qkv is less than a row or no multiple of 8";
  if (a.rot != ROT_NONE && a.rot != ROT_HALVES && a.rot != ROT_NEIGHBOURS) return "unknown rotation";
  if (a.rot != ROT_NONE) {
    if (a.rot_dim < 16 || a.rot_dim > c.DH || a.rot_dim % 16) return "rot_dim is a multiple of 16 up to the head width";
    if (!a.cs || (uintptr_t)a.cs % 16) return "a rotation needs its table, 16-byte aligned";
  }
  for (int g = 0; g < c.G; ++g) {
    if (!a.qkv[g] || (uintptr_t)a.qkv[g] % 16) return "qkv is NULL or not 16-byte aligned";
    if (a.has_q && (!a.q[g] || (uintptr_t)a.q[g] % 16)) return "q is NULL or not 16-byte aligned";
  }
  if (a.has_q && (a.ld_q % 8 || (int64_t)a.ld_q < (int64_t)a.H * c.DH)) return "ld_q is less than a row or no multiple of 8";
  return nullptr;
}

// Threads per page and head: as many as it can have units of new rows, in powers of two, 256 with up to four units each beyond that.  Idle waves
// cost: 301 tokens at most of 16 sequences in pages of 32 rows of 64 (128 units) take 12.5 us with 128 threads, 14.5 with 256.
hipError_t launch_append(const AppendArgs& args, hipStream_t s) {
  AppendArgs a = args;
  const CacheArgs& c = a.c;
  if (a.rot == ROT_NONE) a.rot_dim = 0;
  const int upr = c.DH / 16, rows = c.max_q < c.page ? c.max_q : c.page;
  const int nt = rows * upr <= 64 ? 64 : rows * upr <= 128 ? 128 : 256, upt = (rows * upr + nt - 1) / nt;
  const int64_t pages = (c.max_q + c.page - 2) / c.page + 1;
  const int64_t cache_blocks = pages * 2 * c.HKV;
  const int64_t q_blocks = a.has_q ? ((int64_t)c.max_q * a.H * upr + nt - 1) / nt : 0;
  if (cache_blocks + q_blocks > 0x7fffffffLL || (int64_t)c.max_q * a.H * upr > 0x7fffff00LL) return hipErrorInvalidValue;
  a.cache_blocks = (int)cache_blocks;
  const dim3 grid((unsigned)(cache_blocks + q_blocks), c.B, c.G);
  if (c.kind == CACHE_INT8) run_append<CACHE_INT8>(a, grid, nt, upt, s);
  else run_append<CACHE_E4M3>(a, grid, nt, upt, s);
  return hipGetLastError();
}

}  // namespace hydra
