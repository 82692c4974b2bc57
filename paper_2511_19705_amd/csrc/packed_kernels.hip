// Products with weights whose codes are packed to four bits:
//   Y[t][o] = sum_c s[o][c / g] q[o][c] x[t][c],   x float32, bfloat16, or 8 bits with scales of its own.
// The packed copy holds the codes in the order in which a lane of the matrix instructions takes them (pack_kernel), and each
// row tile's scales behind each other.  Codes reach the matrix cores as 16 q: a nibble in the upper half of a byte is its
// signed value times 16, so that two masks and a shift unpack eight of them, and the result is multiplied by 1 / 16 (exact) at
// the end.  With 8-bit activations the sums over a group are exact integers; with float32 ones the activations are taken in
// three bfloat16 parts, exactly.
#include "cafeq_common.hpp"
#include "cafeq_internal.hpp"
#include "packed.hpp"

namespace cafeq {
namespace {

// One thread a lane's 16 bytes: row tile, 128 columns, lane.
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

// A workgroup owns 16 rows of the weight and 16 TT tokens; its waves share the columns, 128 at a time, and add up through LDS.
// v_mfma 16x16: A the codes (16 rows), B the activations (16 tokens): a lane has four rows of one token, whose scales are one
// 16-byte load.  Sums start anew every FG columns (the common divisor of both groups and 128) and are taken up in float32 with
// their scales.
template <class X, int TT, int FG>
__global__ __launch_bounds__(1024) void packed_small_kernel(const PackedCall a) {
  extern __shared__ float red[];
  const int tid = threadIdx.x, lane = tid & 63, nwave = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, kq = lane >> 4;
  const int64_t rt = blockIdx.x, t0 = int64_t(blockIdx.y) * 16 * TT;
  const int nkb = int(a.p.kblocks), kb0 = wave * nkb / nwave, kb1 = (wave + 1) * nkb / nwave;
  const uint4* w = reinterpret_cast<const uint4*>(a.packed) + (rt * nkb) * 64 + lane;
  const float* sw = reinterpret_cast<const float*>(a.packed + a.p.scales_at) + rt * a.p.groups * kRowTile + kq * 4;
  f32x4 y[TT];
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) y[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int UPB = kBlockK / FG;                 // units a block of 128 columns
  int wu = kb0 * UPB % a.wunits, wg = kb0 * UPB / a.wunits;
  int xu = X::kScaled ? kb0 * UPB % a.xunits : 0, xg = X::kScaled ? kb0 * UPB / a.xunits : 0;
  for (int kb = kb0; kb < kb1; ++kb) {
    const uint4 q = w[int64_t(kb) * 64];
    const uint32_t qd[4] = {q.x, q.y, q.z, q.w};
    typename X::Chunk xv[TT][2];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt) {
      const int64_t t = t0 + tt * 16 + l16;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t k = int64_t(kb) * kBlockK + 64 * j + 16 * kq;
        xv[tt][j] = X::load(a.x, t * a.ldx + k, t < a.n && k < a.p.cols);
      }
    }
#pragma unroll
    for (int u = 0; u < UPB; ++u) {
      const f32x4 s4 = *reinterpret_cast<const f32x4*>(sw + int64_t(min(wg, int(a.p.groups) - 1)) * kRowTile);
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) {
        typename X::Acc acc = {};
        if constexpr (FG == 128) {
          X::mul(acc, qd[0], qd[1], xv[tt][0]);
          X::mul(acc, qd[2], qd[3], xv[tt][1]);
        } else if constexpr (FG == 64) {
          X::mul(acc, qd[2 * u], qd[2 * u + 1], xv[tt][u]);
        } else {
          // 32 of the 64 columns: the other lanes' activations as zeros
          X::mul(acc, qd[2 * (u >> 1)], qd[2 * (u >> 1) + 1], X::keep(xv[tt][u >> 1], (kq >> 1) == (u & 1)));
        }
        float sx = 1.f;
        if constexpr (X::kScaled) {
          const int64_t t = t0 + tt * 16 + l16;
          sx = t < a.n ? a.xscales[t * a.xgroups + min(xg, int(a.xgroups) - 1)] : 0.f;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) y[tt][r] = fmaf(X::value(acc, r) * sx, s4[r], y[tt][r]);
      }
      if (++wu == a.wunits) { wu = 0; ++wg; }
      if constexpr (X::kScaled) if (++xu == a.xunits) { xu = 0; ++xg; }
    }
  }
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) *reinterpret_cast<f32x4*>(&red[((wave * TT + tt) * 64 + lane) * 4]) = y[tt];
  __syncthreads();
  // value e: token e / 16, row e % 16
  for (int e = tid; e < 256 * TT; e += blockDim.x) {
    const int o = e & 15, tok = e >> 4;
    const int64_t t = t0 + tok, row = rt * kRowTile + o;
    const int at = (((tok >> 4) * 64) + (o >> 2) * 16 + (tok & 15)) * 4 + (o & 3);
    float v = 0.f;
    for (int i = 0; i < nwave; ++i) v += red[i * TT * 256 + at];
    if (t < a.n && row < a.p.rows) store_y(a.y, a.ydtype, t * a.ldy + row, v * 0.0625f);
  }
}

template <class X, int TT>
int launch_small_tt(const PackedCall& a, hipStream_t st) {
  const int64_t nkb = a.p.kblocks;
  const int nw = int(std::min<int64_t>(16, std::max<int64_t>(1, nkb / 2)));
  const dim3 grid(unsigned((a.p.rows + kRowTile - 1) / kRowTile), unsigned((a.n + 16 * TT - 1) / (16 * TT)));
  const size_t lds = size_t(nw) * TT * 1024;
  switch (a.fg) {
    case 128: hipLaunchKernelGGL((packed_small_kernel<X, TT, 128>), grid, dim3(nw * 64), lds, st, a); break;
    case 64: hipLaunchKernelGGL((packed_small_kernel<X, TT, 64>), grid, dim3(nw * 64), lds, st, a); break;
    default: hipLaunchKernelGGL((packed_small_kernel<X, TT, 32>), grid, dim3(nw * 64), lds, st, a); break;
  }
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

template <class X>
int launch_small(const PackedCall& a, hipStream_t st) {
  return a.n <= 16 ? launch_small_tt<X, 1>(a, st) : launch_small_tt<X, 2>(a, st);
}

// Whether the products run in tiles of many tokens.
bool by_tiles(int64_t n) { return n > 64; }

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
  return by_tiles(n) ? packed_gemm_bytes(x_type, n, p) : 0;
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
  const int64_t gx = x_type != CAFEQ_I8 || xgroup == 0 ? in : xgroup;
  if (gx < 32 || gx % 32 != 0 || in % gx != 0) return CAFEQ_ERR_BAD_SHAPE;
  const int size = x_type == CAFEQ_F32 ? 4 : x_type == CAFEQ_BF16 ? 2 : 1;
  if (n > (int64_t(1) << 20) || ldx > (int64_t(1) << 24)) return CAFEQ_ERR_UNSUPPORTED;   // a tile's offsets stay below 2^32 bytes
  if (!aligned16(X) || !aligned16(packed) || ldx * size % 16 != 0 || (reinterpret_cast<uintptr_t>(Y) & (y_dtype == CAFEQ_F32 ? 3u : 1u)) != 0 ||
      (reinterpret_cast<uintptr_t>(xscales) & 3u) != 0)
    return CAFEQ_ERR_BAD_ALIGN;
  if (n == 0) return CAFEQ_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto step = [in](int64_t g) { return g == in || g % 128 == 0 ? 128 : g % 64 == 0 ? 64 : 32; };
  const int fg = std::min(step(p.group), step(gx));
  const PackedCall c{static_cast<const uint8_t*>(packed), p, X, x_type, n, ldx, xscales, in / gx, fg, int((p.group + fg - 1) / fg),
                     int((gx + fg - 1) / fg), Y, ldy, y_dtype};
  if (by_tiles(n)) {
    if (!ws && packed_gemm_bytes(x_type, n, p)) return CAFEQ_ERR_WORKSPACE;
    if (!aligned16(ws)) return CAFEQ_ERR_BAD_ALIGN;
    return launch_packed_gemm(c, ws, st);
  }
  switch (x_type) {
    case CAFEQ_I8: return launch_small<XI8>(c, st);
    case CAFEQ_BF16: return launch_small<XBf16>(c, st);
    default: return launch_small<XF32>(c, st);
  }
}

}  // extern "C"
