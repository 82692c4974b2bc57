// Products with weights whose codes are packed to four bits:
//   Y[t][o] = sum_c s[o][c / g] q[o][c] x[t][c],   x float32, bfloat16, or 8 bits with scales of its own.
// The packed copy holds the codes in the order in which a lane of the matrix instructions takes them (pack_kernel), and each
// row tile's scales behind each other.  Codes reach the matrix cores as 16 q: a nibble in the upper half of a byte is its
// signed value times 16, so that two masks and a shift unpack eight of them, and the result is multiplied by 1 / 16 (exact) at
// the end.  With 8-bit activations the sums over a unit of at most 128 columns are exact integers; with float32 ones the activations are taken in
// three bfloat16 parts, exactly.
#include "cafeq_common.hpp"
#include "cafeq_internal.hpp"
#include "packed.hpp"

namespace cafeq {
namespace {

// One thread a lane's 16 bytes: row tile, 128 columns, lane.  Run once for a weight: 36864 x 4608 70 us (3.7 TB/s; a lane's reads of eight codes
// lie a row apart).
__global__ __launch_bounds__(256) void pack_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales, PackedShape p,
                                                   uint8_t* __restrict__ packed) {
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t total = p.row_tiles * p.kblocks * 64;
  if (id < total) {
    const int lane = int(id & 63), kb = int(id / 64 % p.kblocks);
    const int64_t row = id / 64 / p.kblocks * kRowTile + (lane & 15);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {      // dword i: pair i / 2, eight columns
      const int64_t k = int64_t(kb) * kBlockK + 64 * (i >> 1) + 16 * (lane >> 4) + 8 * (i & 1);
      w[i] = 0u;
      if (row < p.rows && k < p.cols) {
        const int8_t* q = codes + row * p.cols + k;
#pragma unroll
        for (int b = 0; b < 4; ++b) w[i] |= (uint32_t(q[b]) & 15u) << (8 * b) | (uint32_t(q[4 + b]) & 15u) << (8 * b + 4);
      }
    }
    reinterpret_cast<uint4*>(packed)[id] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  float* out = reinterpret_cast<float*>(packed + p.scales_at);
  const int64_t nscale = p.row_tiles * p.groups * kRowTile, step = int64_t(gridDim.x) * 256;
  for (int64_t i = id; i < nscale; i += step) {
    const int64_t g = i / kRowTile % p.groups, row = i / kRowTile / p.groups * kRowTile + i % kRowTile;
    out[i] = row < p.rows ? scales[row * p.groups + g] : 0.f;
  }
}

// A workgroup owns 16 OT rows of the weight and 16 TT tokens; its waves share the columns, each a run of blocks of 128, and add up
// through LDS in order.  v_mfma 16x16: A the codes (16 rows), B the activations (16 tokens): a lane has four rows of one token, whose
// scales are one 16-byte load.  Sums start anew every FG columns (the common divisor of both groups and 128) and are taken up in
// float32 with their scales.  A wave requests U blocks at once (weights, activations, scales) before it multiplies the first: with few
// tokens nothing but the bytes in flight counts.  Weights from memory / from the memory-side cache of 256 MB, us: one token of 8 bits, 36864 x 4608
// 22.0 / 17.0 (4.1 / 5.3 TB/s), 3584 x 14336 9.3 / 7.5; in bfloat16 28.0 / 21.2 and 11.5 / 9.2; 16 tokens of 8 bits 26.0 / 22.5 and 14.9 / 14.1 (every
// row tile reads their activations from L2).  float32 67 and 23: every row tile splits its activations anew, and one token's fill one of 16 columns.
template <class X, int TT, int OT, int FG>
__global__ __launch_bounds__(1024) void packed_small_kernel(const PackedCall a) {
  extern __shared__ float red[];
  constexpr int UPB = kBlockK / FG;                 // units of a block
  constexpr int U = TT * OT > 1 || FG == 32 ? 1 : 2;   // blocks requested at once
  const int tid = threadIdx.x, lane = tid & 63, nwave = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, kq = lane >> 4;
  const int rt0 = blockIdx.x * OT, t0 = blockIdx.y * 16 * TT;
  const int nkb = int(a.p.kblocks), kb0 = wave * nkb / nwave, kb1 = (wave + 1) * nkb / nwave;
  const int cols = int(a.p.cols), ngroup = int(a.p.groups), nxgroup = int(a.xgroups);
  const uint4* w[OT];
  const float* sw[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) {
    const int64_t rt = min(rt0 + o, int(a.p.row_tiles) - 1);
    w[o] = reinterpret_cast<const uint4*>(a.packed) + rt * nkb * 64 + lane;
    sw[o] = reinterpret_cast<const float*>(a.packed + a.p.scales_at) + rt * ngroup * kRowTile + kq * 4;
  }
  const void* xp[TT];
  const float* sxp[TT];
  bool live[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int64_t tok = t0 + 16 * t + l16;
    live[t] = tok < a.n;
    xp[t] = static_cast<const char*>(a.x) + (live[t] ? tok : 0) * a.ldx * X::kSize;
    sxp[t] = X::kScaled ? a.xscales + (live[t] ? tok : 0) * a.xgroups : nullptr;
  }
  f32x4 y[OT][TT];
#pragma unroll
  for (int o = 0; o < OT; ++o)
#pragma unroll
    for (int t = 0; t < TT; ++t) y[o][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kb = kb0; kb < kb1; kb += U) {
    uint4 q[U][OT];
    typename X::Chunk xv[U][TT][2];
    f32x4 s4[U][UPB][OT];
    float sx[U][UPB][TT];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (kb + i < kb1) {
#pragma unroll
        for (int o = 0; o < OT; ++o) q[i][o] = w[o][(kb + i) * 64];
      }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (kb + i < kb1) {
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int k = (kb + i) * kBlockK + 64 * j + 16 * kq;
            xv[i][t][j] = X::load(xp[t], k, live[t] && k < cols);
          }
#pragma unroll
        for (int u = 0; u < UPB; ++u) {
          const int unit = (kb + i) * UPB + u;
          const int wg = min(unit_group(unit, a.wunits, a.winv), ngroup - 1);
#pragma unroll
          for (int o = 0; o < OT; ++o) s4[i][u][o] = *reinterpret_cast<const f32x4*>(sw[o] + wg * kRowTile);
          if constexpr (X::kScaled) {
            const int xg = min(unit_group(unit, a.xunits, a.xinv), nxgroup - 1);
#pragma unroll
            for (int t = 0; t < TT; ++t) sx[i][u][t] = sxp[t][xg];
          }
        }
      }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (kb + i < kb1) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          typename X::Form xf[2];
          X::form(xf[0], xv[i][t][0]);
          X::form(xf[1], xv[i][t][1]);
#pragma unroll
          for (int o = 0; o < OT; ++o) {
            const uint4& c = q[i][o];
#pragma unroll
            for (int u = 0; u < UPB; ++u) {
              typename X::Acc acc = {};
              if constexpr (FG == 128) {
                X::mul(acc, c.x, c.y, xf[0]);
                X::mul(acc, c.z, c.w, xf[1]);
              } else if constexpr (FG == 64) {
                X::mul(acc, u ? c.z : c.x, u ? c.w : c.y, xf[u]);
              } else {
                X::mul_in(acc, u >> 1 ? c.z : c.x, u >> 1 ? c.w : c.y, xf[u >> 1], (kq >> 1) == (u & 1));   // 32 of 64 columns
              }
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float v = X::value(acc, r);
                if constexpr (X::kScaled) v *= sx[i][u][t];
                y[o][t][r] = fmaf(v, s4[i][u][o][r], y[o][t][r]);
              }
            }
          }
        }
      }
  }
#pragma unroll
  for (int o = 0; o < OT; ++o)
#pragma unroll
    for (int t = 0; t < TT; ++t) *reinterpret_cast<f32x4*>(&red[(((wave * OT + o) * TT + t) * 64 + lane) * 4]) = y[o][t];
  __syncthreads();
  // value e: token e / (16 OT), row e % (16 OT)
  for (int e = tid; e < 256 * OT * TT; e += blockDim.x) {
    const int o = e & 15, ot = (e >> 4) % OT, tok = (e >> 4) / OT;
    const int at = ((ot * TT + (tok >> 4)) * 64 + (o >> 2) * 16 + (tok & 15)) * 4 + (o & 3);
    const int64_t row = int64_t(rt0 + ot) * kRowTile + o;
    float v = 0.f;
    for (int i = 0; i < nwave; ++i) v += red[i * OT * TT * 256 + at];
    if (t0 + tok < a.n && row < a.p.rows) store_y(a.y, a.ydtype, (t0 + tok) * a.ldy + row, v * code_unit(X::kScaled));
  }
}

template <class X, int TT, int OT>
int launch_small_tt(const PackedCall& a, hipStream_t st) {
  const int nkb = int(a.p.kblocks);
  const unsigned gx = unsigned((a.p.rows + kRowTile * OT - 1) / (kRowTile * OT)), gy = unsigned((a.n + 16 * TT - 1) / (16 * TT));
  // Sixteen waves a compute unit; no more of them to a workgroup than that takes (36864 x 4608, one token, 16 / 4 waves: 23 / 16.5 us), as many
  // where rows are few (3584 x 14336, 4 / 16: 9.7 / 7.6)
  int nw = 16 / OT;
  while (nw > 1 && (int64_t(gx) * gy * (nw / 2) >= 16 * device_cu_count() || nkb < nw * 2)) nw /= 2;
  const dim3 grid(gx, gy);
  const size_t lds = size_t(nw) * OT * TT * 1024;
  switch (a.fg) {
    case 128: hipLaunchKernelGGL((packed_small_kernel<X, TT, OT, 128>), grid, dim3(nw * 64), lds, st, a); break;
    case 64: hipLaunchKernelGGL((packed_small_kernel<X, TT, OT, 64>), grid, dim3(nw * 64), lds, st, a); break;
    default: hipLaunchKernelGGL((packed_small_kernel<X, TT, OT, 32>), grid, dim3(nw * 64), lds, st, a); break;
  }
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

// Two row tiles a wave share its activations, whose way from L2 then weighs less (8 bits, 36864 x 4608, 16 tokens: 30 -> 23.5 us), where the
// workgroups still fill the chip (3584 x 14336: 13.6 -> 17); float activations of two row or token tiles leave too few registers
// (bfloat16, 36864 x 4608, 8 tokens: 31 -> 52).
int launch_small(const PackedCall& a, hipStream_t st) {
  const bool many = a.p.row_tiles >= 4 * device_cu_count();
  if (a.x_type == CAFEQ_I8) {
    if (a.n <= 16) return many && a.n > 2 ? launch_small_tt<XI8, 1, 2>(a, st) : launch_small_tt<XI8, 1, 1>(a, st);
    return many ? launch_small_tt<XI8, 2, 2>(a, st) : launch_small_tt<XI8, 2, 1>(a, st);
  }
  if (a.x_type == CAFEQ_BF16) return a.n <= 16 ? launch_small_tt<XBf16, 1, 1>(a, st) : launch_small_tt<XBf16, 2, 1>(a, st);
  return launch_small_tt<XF32, 1, 1>(a, st);
}

// Whether the products run in tiles of 32 and more tokens.  Few tokens do not: every wave has its own run of columns there, without a stage's
// barriers, but the weights are read again for every 16 or 32 tokens.  us this way / in tiles: 8 bits, 2048 x 4608 and 64 tokens 8 / 12, 96 13.5 / 13,
// 3584 x 14336 and 24 19 / 17, 64 25 / 19; bfloat16, 2048 x 4608 and 64 tokens 11 / 14, 128 19 / 15, 36864 x 4608 and 8 31 / 33, 16 43 / 33; float32,
// 2048 x 4608 and 64 21 / 24, 3584 x 14336 and 32 55 / 34.
bool by_tiles(int x_type, int64_t n, const PackedShape& p) {
  return n > (x_type == CAFEQ_I8 ? 16 : 8) && double(n) * double(p.rows) * double(p.cols) > 0.9e9;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_packed_bytes(int64_t out, int64_t in, int64_t group) {
  PackedShape p;
  return packed_shape(out, in, group, &p) == CAFEQ_OK ? size_t(p.bytes) : 0;
}

int cafeq_pack_nibbles(const int8_t* codes, const float* scales, int64_t out, int64_t in, int64_t group, void* packed, void* stream) {
  if (!codes || !scales || !packed) return CAFEQ_ERR_INVALID_ARG;
  PackedShape p;
  const int rc = packed_shape(out, in, group, &p);
  if (rc) return rc;
  if (!aligned16(packed) || (reinterpret_cast<uintptr_t>(scales) & 3u) != 0) return CAFEQ_ERR_BAD_ALIGN;
  const int64_t n = p.row_tiles * p.kblocks * 64;
  hipLaunchKernelGGL(pack_kernel, dim3(unsigned((n + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream), codes, scales, p,
                     static_cast<uint8_t*>(packed));
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

size_t cafeq_infer_packed_workspace_bytes(int x_type, int64_t n, int64_t out, int64_t in, int64_t group) {
  PackedShape p;
  if (n < 1 || x_type < CAFEQ_F32 || x_type > CAFEQ_I8 || packed_shape(out, in, group, &p) != CAFEQ_OK) return 0;
  return by_tiles(x_type, n, p) ? packed_gemm_bytes(x_type, n, p) : 0;
}

int cafeq_infer_packed(const void* X, int x_type, int64_t n, int64_t ldx, const float* xscales, int64_t xgroup, const void* packed,
                       int64_t out, int64_t in, int64_t group, void* Y, int y_dtype, int64_t ldy, void* ws, void* stream) {
  if (!X || !packed || !Y) return CAFEQ_ERR_INVALID_ARG;
  if (x_type != CAFEQ_F32 && x_type != CAFEQ_BF16 && x_type != CAFEQ_I8) return CAFEQ_ERR_INVALID_ARG;
  if (y_dtype != CAFEQ_F32 && y_dtype != CAFEQ_BF16) return CAFEQ_ERR_INVALID_ARG;
  if ((x_type == CAFEQ_I8) != (xscales != nullptr)) return CAFEQ_ERR_INVALID_ARG;
  PackedShape p;
  const int rc = packed_shape(out, in, group, &p);
  if (rc) return rc;
  if (n < 0 || ldx < in || ldy < out) return CAFEQ_ERR_BAD_SHAPE;
  if (n == 1) ldx = in;   // a single row has no next one
  const int64_t gx = x_type != CAFEQ_I8 || xgroup == 0 ? in : xgroup;
  if (gx < 32 || gx % 32 != 0 || in % gx != 0) return CAFEQ_ERR_BAD_SHAPE;
  const int size = x_type == CAFEQ_F32 ? 4 : x_type == CAFEQ_BF16 ? 2 : 1;
  if (n > (int64_t(1) << 19) || ldx > (int64_t(1) << 24)) return CAFEQ_ERR_UNSUPPORTED;   // a grid's rows below 2^16, a tile's offsets below 2^32 bytes
  if (!aligned16(X) || !aligned16(packed) || ldx * size % 16 != 0 || (reinterpret_cast<uintptr_t>(Y) & (y_dtype == CAFEQ_F32 ? 3u : 1u)) != 0 ||
      (reinterpret_cast<uintptr_t>(xscales) & 3u) != 0)
    return CAFEQ_ERR_BAD_ALIGN;
  if (n == 0) return CAFEQ_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto step = [in](int64_t g) { return g == in || g % 128 == 0 ? 128 : g % 64 == 0 ? 64 : 32; };
  const int fg = std::min(step(p.group), step(gx));
  const int wunits = int((p.group + fg - 1) / fg), xunits = int((gx + fg - 1) / fg);
  const PackedCall c{static_cast<const uint8_t*>(packed), p, X, x_type, n, ldx, xscales, in / gx, fg, wunits, xunits, unit_inverse(wunits),
                     unit_inverse(xunits), Y, ldy, y_dtype};
  if (by_tiles(x_type, n, p)) {
    if (!ws && packed_gemm_bytes(x_type, n, p)) return CAFEQ_ERR_WORKSPACE;
    if (!aligned16(ws)) return CAFEQ_ERR_BAD_ALIGN;
    return launch_packed_gemm(c, ws, st);
  }
  return launch_small(c, st);
}

}  // extern "C"
