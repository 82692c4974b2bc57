// Packed 4-bit weights: the layout, and the activations' forms on the matrix cores.
#pragma once
#include "cafeq_common.hpp"

namespace cafeq {

using i32x4 = __attribute__((__vector_size__(4 * sizeof(int)))) int;
using f32x4 = __attribute__((__vector_size__(4 * sizeof(float)))) float;
using bf16x8_t = __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16;

// Codes: tiles of 16 rows x 128 columns, 1 KB each, [row tile][block of 128 columns][lane][16 bytes].  Lane l of a tile holds row
// l % 16 and, in pair j of its two eight-byte pairs, the columns 64 j + 16 (l / 16) + 0 .. 15; byte b of dword e of a pair holds
// column 8 e + b in its lower half and 8 e + 4 + b in its upper one.  A wave's load of a tile is 1 KB side by side, and a lane's
// pair unpacks to 16 consecutive columns, the K range of the 8-bit matrix instructions' lane.
// Scales behind them: [row tile][group][16 rows] float32.  Rows beyond the matrix and columns beyond its width are zeros.
constexpr int kRowTile = 16, kBlockK = 128;

struct PackedShape {
  int64_t rows, cols, group, groups, row_tiles, kblocks, scales_at, bytes;
};

inline int packed_shape(int64_t out, int64_t in, int64_t group, PackedShape* p) {
  if (out < 1 || in < 32 || in % 32 != 0 || group < 0) return CAFEQ_ERR_BAD_SHAPE;
  const int64_t g = group == 0 ? in : group;
  if (g % 32 != 0 || in % g != 0) return CAFEQ_ERR_BAD_SHAPE;
  if (in > 65536 || out > (int64_t(1) << 24)) return CAFEQ_ERR_UNSUPPORTED;   // a row has at most 2048 units, as unit_group() needs
  p->rows = out;
  p->cols = in;
  p->group = g;
  p->groups = in / g;
  p->row_tiles = (out + 2 * kRowTile - 1) / (2 * kRowTile) * 2;   // whole tiles of 32 rows
  p->kblocks = (in + kBlockK - 1) / kBlockK;
  if (p->row_tiles * p->kblocks > (int64_t(1) << 25)) return CAFEQ_ERR_UNSUPPORTED;            // a launch's threads stay below 2^32
  p->scales_at = p->row_tiles * p->kblocks * 1024;
  p->bytes = p->scales_at + p->row_tiles * p->groups * kRowTile * int64_t(sizeof(float));
  return CAFEQ_OK;
}

// The group of a unit, unit / units, by a product: units are at most 2048, where ceil(2^32 / units) is exact enough for whole quotients
inline uint32_t unit_inverse(int units) { return units > 1 ? uint32_t(((uint64_t(1) << 32) + units - 1) / units) : 0u; }
__device__ __forceinline__ int unit_group(int unit, int units, uint32_t inv) { return units > 1 ? int(__umulhi(uint32_t(unit), inv)) : unit; }

// A checked call of cafeq_infer_packed
struct PackedCall {
  const uint8_t* packed;
  PackedShape p;
  const void* x;
  int x_type;
  int64_t n, ldx;
  const float* xscales;   // [n][xgroups], 8-bit activations
  int64_t xgroups;
  int fg;                 // columns a unit: sums start anew there and take their scales
  int wunits, xunits;     // units a scale of the weights, of the activations
  uint32_t winv, xinv;    // their unit_inverse()
  void* y;
  int64_t ldy;
  int ydtype;
};
// packed_gemm.hip: many tokens
size_t packed_gemm_bytes(int x_type, int64_t n, const PackedShape& p);
int launch_packed_gemm(const PackedCall& c, void* ws, hipStream_t st);

__device__ __forceinline__ uint32_t low16(uint32_t w) { return (w << 4) & 0xF0F0F0F0u; }   // 16 q of columns 0 .. 3 of a dword
__device__ __forceinline__ uint32_t high16(uint32_t w) { return w & 0xF0F0F0F0u; }         // of columns 4 .. 7

// Codes of columns I and I + 1 of a dword's eight (w: the dword, or the dword >> 4 for the upper four) as a pair of bfloat16, each divided by
// 16, exactly: the hardware's conversion of a signed nibble gives q / 16.
template <int I>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w) {
  uint32_t a, b;
  if constexpr (I == 0) {
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(a) : "v"(w));
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(b) : "v"(w));
  } else {
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(a) : "v"(w));
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(b) : "v"(w));
  }
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
// eight codes / 16 as a bfloat16 operand
__device__ __forceinline__ bf16x8_t bf16_codes(uint32_t w) {
  const uint32_t hi = w >> 4;
  union { uint32_t u[4]; bf16x8_t v; } f;
  f.u[0] = bf16_pair<0>(w); f.u[1] = bf16_pair<2>(w); f.u[2] = bf16_pair<0>(hi); f.u[3] = bf16_pair<2>(hi);
  return f.v;
}
// what a result is multiplied by in the end: 8-bit operands hold 16 q, bfloat16 ones q / 16
__host__ __device__ inline float code_unit(bool i8) { return i8 ? 0.0625f : 16.f; }

// two float32 values' leading bits as a pair of bfloat16, and what they leave (nothing of an infinity)
__device__ __forceinline__ uint32_t split_pair(float& a, float& b) {
  const uint32_t ha = __float_as_uint(a) & 0xFFFF0000u, hb = __float_as_uint(b) & 0xFFFF0000u;
  const float fa = __uint_as_float(ha), fb = __uint_as_float(hb);
  const uint32_t p = __builtin_amdgcn_perm(hb, ha, 0x07060302u);
  a = a == fa ? 0.f : a - fa;
  b = b == fb ? 0.f : b - fb;
  return p;
}

__device__ __forceinline__ void store_y(void* y, int dtype, int64_t at, float v) {
  if (dtype == CAFEQ_F32) static_cast<float*>(y)[at] = v;
  else static_cast<uint16_t*>(y)[at] = bf16_bits(v);
}

// The forms of the activations.  Chunk: 16 consecutive columns of a token (a lane's share of 64) as loaded; Form: as the matrix
// instructions take them; mul: 64 columns of 16 rows times 16 tokens onto acc, the weights' two dwords of the same columns; mul_in: of the
// lanes for which `in` is set only.  The others have codes of zero where the products are integers; where they are floats it is the
// activations that are zero there: an infinity times a code of zero would be no number.
struct XI8 {
  static constexpr bool kScaled = true;
  static constexpr int kSize = 1;
  using Acc = i32x4;
  using Chunk = i32x4;
  using Form = i32x4;
  static __device__ __forceinline__ Chunk load(const void* x, int at, bool in) {
    return in ? *reinterpret_cast<const i32x4*>(static_cast<const int8_t*>(x) + at) : i32x4{0, 0, 0, 0};
  }
  static __device__ __forceinline__ void form(Form& f, const Chunk& c) { f = c; }
  static __device__ __forceinline__ void mul(Acc& acc, uint32_t w0, uint32_t w1, const Form& f) {
    const i32x4 a = {int(low16(w0)), int(high16(w0)), int(low16(w1)), int(high16(w1))};
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, f, acc, 0, 0, 0);
  }
  static __device__ __forceinline__ void mul_in(Acc& acc, uint32_t w0, uint32_t w1, const Form& f, bool in) {
    mul(acc, in ? w0 : 0u, in ? w1 : 0u, f);
  }
  static __device__ __forceinline__ float value(const Acc& acc, int r) { return float(acc[r]); }
};

struct XBf16 {
  static constexpr bool kScaled = false;
  static constexpr int kSize = 2;
  using Acc = f32x4;
  struct Chunk { bf16x8_t v[2]; };
  using Form = Chunk;
  static __device__ __forceinline__ Chunk load(const void* x, int at, bool in) {
    Chunk c;
    const bf16x8_t* p = reinterpret_cast<const bf16x8_t*>(static_cast<const uint16_t*>(x) + at);
    c.v[0] = in ? p[0] : bf16x8_t{};
    c.v[1] = in ? p[1] : bf16x8_t{};
    return c;
  }
  static __device__ __forceinline__ void form(Form& f, const Chunk& c) { f = c; }
  static __device__ __forceinline__ void mul(Acc& acc, uint32_t w0, uint32_t w1, const Form& f) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_codes(w0), f.v[0], acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_codes(w1), f.v[1], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ void mul_in(Acc& acc, uint32_t w0, uint32_t w1, const Form& f, bool in) {
    Form g;
#pragma unroll
    for (int e = 0; e < 2; ++e) g.v[e] = in ? f.v[e] : bf16x8_t{};
    mul(acc, w0, w1, g);
  }
  static __device__ __forceinline__ float value(const Acc& acc, int r) { return acc[r]; }
};

struct XF32 {
  static constexpr bool kScaled = false;
  static constexpr int kSize = 4;
  using Acc = f32x4;
  struct Chunk { float v[16]; };
  struct Form { bf16x8_t v[2][3]; };   // three parts of every activation, hi + mid + lo exactly (down to bfloat16's 2^-133)
  static __device__ __forceinline__ Chunk load(const void* x, int at, bool in) {
    Chunk c;
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(x) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = in ? p[i] : make_float4(0.f, 0.f, 0.f, 0.f);
      c.v[4 * i] = f.x; c.v[4 * i + 1] = f.y; c.v[4 * i + 2] = f.z; c.v[4 * i + 3] = f.w;
    }
    return c;
  }
  static __device__ __forceinline__ void form(Form& f, const Chunk& c) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float r[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = c.v[8 * e + i];
#pragma unroll
      for (int s = 0; s < 3; ++s) {
        union { uint32_t u[4]; bf16x8_t v; } part;
#pragma unroll
        for (int i = 0; i < 4; ++i) part.u[i] = split_pair(r[2 * i], r[2 * i + 1]);
        f.v[e][s] = part.v;
      }
    }
  }
  static __device__ __forceinline__ void mul(Acc& acc, uint32_t w0, uint32_t w1, const Form& f) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const bf16x8_t w = bf16_codes(e ? w1 : w0);
#pragma unroll
      for (int s = 2; s >= 0; --s) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, f.v[e][s], acc, 0, 0, 0);   // the small parts first
    }
  }
  static __device__ __forceinline__ void mul_in(Acc& acc, uint32_t w0, uint32_t w1, const Form& f, bool in) {
    Form g;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int s = 0; s < 3; ++s) g.v[e][s] = in ? f.v[e][s] : bf16x8_t{};
    mul(acc, w0, w1, g);
  }
  static __device__ __forceinline__ float value(const Acc& acc, int r) { return acc[r]; }
};

}  // namespace cafeq
