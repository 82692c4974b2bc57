// Attention over the 8-bit cache: what its kernels share.
//
// Products run on the 16-bit matrix instructions with codes as float16 (exact) and transposed: S^T = K Q^T, out^T = V^T P^T.  A column of the
// result is a query row, so that a lane holds scores of one row only, and the scores as they leave the first product are, rounded, what the
// second one takes: nothing moves between lanes.
//
// A page's scale of v, mant 2^exp, goes into the exponent: with y = x + exp (x the score in units of log2) and M the largest y so far, rounded up, less 14,
//   p = 2^(y - M) <= 2^14,   out = sum p mant c_v / sum p 2^-exp.
// What is rounded to float16, p mant in (2^13, 2^15) for the largest (to 11 bits down to 2^-27 of it, to multiples of 2^-37 of it below), so is weighed as it counts in the
// result, however scales differ from page to page; and exp - M is a whole number, so that the exponent's argument takes one rounding, in proportion to itself.
#pragma once
#include "cache.hpp"

namespace cafeq {

using half2_t = __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16;
using half8_t = __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16;
using f32x4_t = __attribute__((__vector_size__(4 * sizeof(float)))) float;
using f32x16_t = __attribute__((__vector_size__(16 * sizeof(float)))) float;

constexpr float kNoKey = -FLT_MAX;       // M before the first key
constexpr float kTop = 14.f;              // log2 of the largest p
constexpr int kRoom = 17;                 // the sum of weights, p 2^-exp, is held in units of 2^(M + kRoom): 2^30 keys of p = 2^14 fit with exp = -100
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kZeroScale = 0x1p-100f;  // pages of v below it hold zeros: their keys have weight, and no value

// Four codes of a dword as float16: 1024 + (q + 128) put together as bits, less 1152; exact.  Five instructions.
__device__ __forceinline__ void half_codes(uint32_t w, half2_t* h) {
  const uint32_t u = w ^ 0x80808080u;
  const half2_t bias = {_Float16(-1152.f), _Float16(-1152.f)};
  h[0] = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + bias;
  h[1] = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + bias;
}
__device__ __forceinline__ half8_t half_codes(uint32_t w0, uint32_t w1) {
  union { half2_t h[4]; half8_t v; } f;
  half_codes(w0, f.h);
  half_codes(w1, f.h + 2);
  return f.v;
}

__device__ __forceinline__ half2_t to_half(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(half2_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}
// out tanh(z); for results of bfloat16, where z comes times 2 log2 e, by the hardware's exponential, good to 2^-22 of `out`
template <bool F32>
__device__ __forceinline__ float capped(float z, float out) {
  if constexpr (F32) return tanhf(z) * out;
  else return fmaf(-2.f * out, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z)), out);
}
// The same for results of bfloat16 under a cap so far above the scores (kWideCap) that 2^-22 of it is more than a score is known to: below a quarter tanh's
// series (the first term left out is below 2^-26 of it), and so good to 2^-20 of itself everywhere.  Float32's tanh serves all caps.
constexpr float kWideCap = 256.f, kNoCap = 0x1p100f;
enum Cap { kCapNone, kCapNear, kCapWide };
__device__ __forceinline__ float capped_wide(float z, float out) {
  const float u = z * (0.5f * kLn2), s = u * u;
  const float series = u * fmaf(s, fmaf(s, fmaf(s, fmaf(s, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
  return fabsf(u) < 0.25f ? series * out : capped<false>(z, out);
}

// The rows of one tile and what of the keys they reach.  Row R of a sequence and key head is token R / rep, query head R % rep of the group.
struct Reach {
  int i, row0;         // sequence, its first row of q
  int len, pos0;       // its tokens; position of its first row
  int rows;            // rows of the sequence and key head that are computed
  int lo, hi;          // keys that any row of the tile reaches
};
__device__ __forceinline__ int key_end(const cafeq_attention& a, int len, int pos) { return a.causal ? min(len, pos + 1) : len; }
__device__ __forceinline__ int key_begin(const cafeq_attention& a, int pos) { return a.window > 0 ? max(0, pos - a.window + 1) : 0; }

__device__ __forceinline__ Reach reach_of(const cafeq_cache& c, const cafeq_attention& a, int i, int rep, int first, int count) {
  Reach r;
  const RowRange rr = rows_of(a.starts, i, int(a.n));
  r.i = i;
  r.row0 = rr.lo;
  r.len = no_room(c, a.starts) ? 0 : tokens_of(c, i);
  r.pos0 = r.len - (rr.hi - rr.lo);
  r.rows = int(min(int64_t(rr.hi - rr.lo), a.longest)) * rep;
  const int last = int(min(unsigned(first) + unsigned(count), unsigned(r.rows))) - 1;
  r.lo = key_begin(a, r.pos0 + first / rep);
  r.hi = last < first ? 0 : key_end(a, r.len, r.pos0 + last / rep);
  return r;
}

// A page's scale of v as mant 2^exp; inv = 2^-(exp + kRoom).  A scale that is no number is its own mantissa.
struct ValueScale { float exp, mant, inv; bool zero; };
__device__ __forceinline__ ValueScale value_scale(float vs) {
  ValueScale s;
  const uint32_t u = __float_as_uint(vs) & 0x7FFFFFFFu, e = u >> 23;
  s.zero = vs < kZeroScale;
  const bool plain = e < 255 && !s.zero;
  s.exp = plain ? float(int(e) - 127) : 0.f;
  s.mant = plain ? __uint_as_float((u & 0x7FFFFFu) | 0x3F800000u) : s.zero ? 0.f : vs;
  // (put together as bits, which the scalar unit does for a wave; subnormal for the largest scales)
  s.inv = !plain ? 1.f / float(1 << kRoom) : __uint_as_float(e < 254u - kRoom ? (254u - kRoom - e) << 23 : 1u << (276u - kRoom - e));
  return s;
}

// Large scores.  The weight's argument is one fused operation, x f - M, while M comes of rounded scores x f: where half a step of the score is one and more the two
// do not fit together (and exp - M is rounded where exp is no whole number).  So where a step of keys may hold scores beyond kFar, a row whose largest one passes kLarge
// takes them against a reference of its own, a whole number that follows the largest one: x' = fl(x f) - base is exact where it counts, and M, o and l go on as they
// are, in units of 2^(base + M).  Rows that meet no such score keep their bits, whatever the rows beside them hold.
constexpr float kFar = 0x1p19f, kLarge = 0x1p12f;
// x f is below kFar for all keys where f is below this: |q| < 2^15, |code| <= 2^7, 64 db channels
constexpr float near_factor(int db) { return kFar / (64.f * db * 0x1p22f); }
// the reference that a row goes on with (0: none), top being its largest score of these keys (kNoKey: none)
__device__ __forceinline__ float next_base(float top, float base, bool first) {
  const bool leaves = base != 0.f ? top > base : fabsf(top) > kLarge && (top > 0.f || first);
  return leaves && top > kNoKey ? ceilf(top) : base;
}
// What a wave's o and l are times in the end, and the M that they are then in units of: a float32 of its own again, base + M + kRoom, however far it is
struct Finish { float all, unit, sum_unit; };
__device__ __forceinline__ Finish finish_of(float M, float base) {
  const float all = base + (M + kRoom), unit = __builtin_amdgcn_exp2f(M - (all - base));
  return {all, unit, unit * float(1 << kRoom)};
}

// Rows of q are taken times a power of two that brings the largest magnitude (its bits) to [2^14, 2^15): bfloat16 then is exact in float16 down to
// 2^-31 of it.  unit: what a product's sum is times, next to the scale of k, in the score (in log2 without a soft cap)
struct QueryScale { float up, unit; };
__device__ __forceinline__ QueryScale query_scale(uint32_t bits, const cafeq_attention& a) {
  const int e = max(-100, int(bits >> 23) - 127);
  QueryScale s;
  s.up = copysignf(bits ? __uint_as_float(uint32_t(127 + 14 - e) << 23) : 1.f, a.scale);      // a negative scale is q's
  s.unit = bits >= 0x7F800000u ? NAN : bits ? ldexpf(fabsf(a.scale), e - 14) : 0.f;
  if (a.softcap <= 0.f) s.unit *= kLog2e;
  return s;
}

// Many rows, by 64 channels (db): keys of a tile, waves of a workgroup (32 rows each), waves a SIMD that registers and LDS allow.  A prompt of 8192, TFLOP/s of the first form:
// 8 heads of 256, 4 waves and 32 keys 675, 8 and 32 817, 8 and 64 856; 16 heads of 128, 4 and 64 817, 8 and 64 849, 4 and 32 (three waves a SIMD) 861, 8 and 128 784;
// 4 heads of 64, 4 and 64 637, 8 and 64 569; in float32 16 heads of 128, 4 and 32 438, 4 and 64 450, 8 and 64 491.
constexpr int many_keys(int dtype, int db) { return db == 2 && dtype != CAFEQ_F32 ? 32 : dtype == CAFEQ_F32 && db > 2 ? 32 : 64; }
constexpr int many_waves(int dtype, int db) { return dtype == CAFEQ_F32 ? (db == 2 ? 8 : 4) : db > 2 ? 8 : 4; }
constexpr int many_resident(int dtype, int db) { return dtype == CAFEQ_F32 ? (db > 2 ? 1 : 2) : db == 1 ? 4 : db == 2 ? 3 : 2; }

struct AttendPlan {
  cafeq_cache c;
  cafeq_attention a;
  int rep, shift;     // query heads of a key head; log2 of the block
  int few_rows;       // sequences with up to so many rows are attend_few's, the others attend_many's
  Units units;        // attend_many: row tiles of all sequences
  int tiles;          // row tiles of a sequence
  int splits, span;   // parts that the keys of a tile may be cut into, steps of 32 keys (attend_many: tiles of keys) in each
  int keep;           // rows of a tile that have room in the parts
  int cap;
  float cap_in, cap_out;      // a score (in log2) under the soft cap: cap_out tanh(score cap_in), cap_in times 2 log2 e for bfloat16
  float* sums;        // parts [sequence][tile][head][split][keep]: (M, sum of weights)
  float* parts;       // and [keep][d]
};

// Four channels of a finished row: v in units of 2^M, divided by the sum of weights
template <class Tag>
__device__ __forceinline__ void store_row(const AttendPlan& p, const Reach& r, int R, int head, int ch, f32x4_t v, float M, float total) {
  const int64_t row = r.row0 + R / p.rep;
  const int h = head * p.rep + R % p.rep;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  typename Tag::elem* y = static_cast<typename Tag::elem*>(p.a.out) + row * p.a.ldo + h * p.a.hso + ch;
  if constexpr (Tag::dtype == CAFEQ_F32) *reinterpret_cast<f32x4_t*>(y) = v * inv;
  else *reinterpret_cast<uint2*>(y) = make_uint2(bf16_bits(v[0] * inv, v[1] * inv), bf16_bits(v[2] * inv, v[3] * inv));
  if (p.a.lse && ch == 0) p.a.lse[row * p.a.heads_q + h] = total == 0.f ? -INFINITY : (M + log2f(total)) * kLn2;
}

int launch_attend_few(const AttendPlan& p, hipStream_t st);
int launch_attend_many(const AttendPlan& p, hipStream_t st);

}  // namespace cafeq
