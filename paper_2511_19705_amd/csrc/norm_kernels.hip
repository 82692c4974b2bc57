// Activations of a quantized layer made ready in 8 bits: residual addition, root-mean-square norm, the blocks of the
// inverse transform (paper Sec. 4.1, the first factor of Y^ = X M^-1 Q(MW)) and a scale per group of columns.
//   h = x + r,  y = h (mean_c h_c^2 + eps)^-1/2 (offset + gain),  z_b = Tinv_b y_b,
//   a_G = max_{c in G} |z_c|,  q = rint(z fl(127 / a)),  s = a / 127.
// Without a transform one workgroup holds a row in registers and reads it once (norm_row_kernel).  With one, that kernel
// leaves 1 / rms of every row and act_tile_kernel forms z from x and r again: a block of z needs the whole row only
// through that one number.
#include "cafeq_common.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kVec = 8;              // consecutive elements a thread owns
constexpr int kMaxThreads = 1024;
constexpr int64_t kMaxRow = int64_t(kMaxThreads) * kVec * 8;
constexpr int kMinGroup = 32;

struct RowArgs {
  const void* x;
  const void* res;
  void* sum;
  int64_t ldx, ldr, lds;
  int64_t d;
  const float* gain;
  float offset, eps;
  int norm;
  int64_t group;          // columns a scale; 0: no codes
  int8_t* codes;          // [n][d]
  float* scales;          // [n][d / group]
  void* values;
  int64_t ldv;
  int vdtype;
  float* rstd;            // [n], or null
};

// |v| as bits: ordered like the magnitudes, infinities above all numbers and NaN above those, so that a group's maximum says
// when the group holds one
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <int LANES>
__device__ __forceinline__ uint32_t cluster_umax(uint32_t v) {
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1) v = max(v, uint32_t(__shfl_xor(int(v), m)));
  return v;
}
__device__ __forceinline__ uint32_t cluster_umax(uint32_t v, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) v = max(v, uint32_t(__shfl_xor(int(v), m)));
  return v;
}

// The grid's reciprocal step; a group with an infinity or a NaN has all codes 0 and that as its scale, so that what reads it
// is not finite either.
__device__ __forceinline__ float act_inv(float a) { return (a > 0.f && a <= FLT_MAX) ? fminf(__fdiv_rn(127.f, a), FLT_MAX) : 0.f; }
__device__ __forceinline__ float act_code(float z, float inv) {
  const float q = __builtin_rintf(__fmul_rn(z, inv));
  return inv > 0.f ? fminf(fmaxf(q, -127.f), 127.f) : 0.f;
}

__device__ __forceinline__ uint16_t bf16_rne(float f) {
  const uint32_t u = __float_as_uint(f);
  return mag_bits(f) > 0x7F800000u ? uint16_t((u >> 16) | 0x40u) : uint16_t((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

template <class Tag, bool ALIGNED>
__device__ __forceinline__ void load_vec(float (&v)[kVec], const void* base, int64_t at, int64_t left) {
  const auto* p = static_cast<const typename Tag::elem*>(base) + at;
  if constexpr (ALIGNED) {
    const float4 a = load4(p), b = load4(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = e < left ? load1(p + e) : 0.f;
  }
}

template <bool ALIGNED>
__device__ __forceinline__ void store_vec(const float (&v)[kVec], void* base, int dtype, int64_t at, int64_t left) {
  if (dtype == CAFEQ_F32) {
    float* p = static_cast<float*>(base) + at;
    if constexpr (ALIGNED) {
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) if (e < left) p[e] = v[e];
    }
  } else {
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    if constexpr (ALIGNED) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = uint32_t(bf16_rne(v[2 * e])) | (uint32_t(bf16_rne(v[2 * e + 1])) << 16);
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) if (e < left) p[e] = bf16_rne(v[e]);
    }
  }
}

// One workgroup a row, the row in registers: CH chunks of eight columns a thread.  Reads x and r once and writes each output
// once; bound by those bytes for long batches and by the launch and one trip to memory for a few rows.
// ALIGNED: every row of every operand starts at a multiple of 16 bytes and d is a multiple of 8.
template <class Tag, int CH, bool ALIGNED>
__global__ __launch_bounds__(kMaxThreads) void norm_row_kernel(const RowArgs a) {
  __shared__ float part[kMaxThreads / kWave];
  __shared__ uint32_t top[kMaxRow / kMinGroup];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nthr = blockDim.x, nwave = nthr >> 6;
  const int64_t row = blockIdx.x, d = a.d;
  float v[CH][kVec];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t at = int64_t(tid + c * nthr) * kVec;
    if (at < d) {
      load_vec<Tag, ALIGNED>(v[c], a.x, row * a.ldx + at, d - at);
      if (a.res) {
        float r[kVec];
        load_vec<Tag, ALIGNED>(r, a.res, row * a.ldr + at, d - at);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[c][e] += r[e];
      }
      if (a.sum) store_vec<ALIGNED>(v[c], a.sum, Tag::dtype, row * a.lds + at, d - at);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[c][e] = 0.f;
    }
  }
  if (a.norm) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < kVec; ++e) s = fmaf(v[c][e], v[c][e], s);
    s = wave_sum(s);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < nwave; ++w) s += part[w];
    const float rstd = 1.f / sqrtf(s / float(d) + a.eps);
    if (a.rstd && tid == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t at = int64_t(tid + c * nthr) * kVec;
      float g[kVec];
      if (a.gain && at < d) {
        load_vec<F32Tag, ALIGNED>(g, a.gain, at, d - at);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[c][e] = v[c][e] * rstd * (a.offset + g[e]);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[c][e] = v[c][e] * rstd;
      }
    }
  }
  if (!a.codes) {
    if (a.values)
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int64_t at = int64_t(tid + c * nthr) * kVec;
        if (at < d) store_vec<ALIGNED>(v[c], a.values, a.vdtype, row * a.ldv + at, d - at);
      }
    return;
  }
  // a thread's eight columns lie in one group: groups are multiples of 32, or the row
  const int ngroup = int(d / a.group), lanes = int(a.group / kVec);
  const bool clusters = a.group <= 512 && (a.group & (a.group - 1)) == 0;
  uint32_t m[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    m[c] = 0u;
#pragma unroll
    for (int e = 0; e < kVec; ++e) m[c] = max(m[c], mag_bits(v[c][e]));
  }
  if (clusters) {
#pragma unroll
    for (int c = 0; c < CH; ++c) m[c] = cluster_umax(m[c], lanes);
  } else {
    // the maximum is the same in whatever order it is formed
    for (int g = tid; g < ngroup; g += nthr) top[g] = 0u;
    __syncthreads();
    if (ngroup == 1) {
      uint32_t w = 0u;
#pragma unroll
      for (int c = 0; c < CH; ++c) w = max(w, m[c]);
      w = cluster_umax<64>(w);
      if (lane == 0) atomicMax(&top[0], w);
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int64_t at = int64_t(tid + c * nthr) * kVec;
        const uint32_t w = cluster_umax<4>(m[c]);
        if ((tid & 3) == 0 && at < d) atomicMax(&top[at / a.group], w);
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t at = int64_t(tid + c * nthr) * kVec;
      if (at < d) m[c] = top[at / a.group];
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int64_t at = int64_t(tid + c * nthr) * kVec;
    if (at >= d) continue;
    const float amax = __uint_as_float(m[c]), inv = act_inv(amax), s = __fdiv_rn(amax, 127.f);
    float q[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) q[e] = act_code(v[c][e], inv);
    int8_t* p = a.codes + row * d + at;
    if constexpr (ALIGNED) {
      *reinterpret_cast<uint2*>(p) = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) if (e < d - at) p[e] = int8_t(int(q[e]));
    }
    if (at % a.group == 0) a.scales[row * ngroup + at / a.group] = s;
    if (a.values) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) q[e] = __fmul_rn(q[e], s);
      store_vec<ALIGNED>(q, a.values, a.vdtype, row * a.ldv + at, d - at);
    }
  }
}

template <class Tag, bool ALIGNED>
int launch_rows_as(const RowArgs& a, int64_t n, hipStream_t st) {
  const int64_t chunks = (a.d + kVec - 1) / kVec;
  int ch = 1;
  while ((chunks + ch - 1) / ch > kMaxThreads) ch *= 2;
  const int t = int(((chunks + ch - 1) / ch + 63) / 64 * 64);
  const dim3 grid{unsigned(n)}, block{unsigned(t)};
  switch (ch) {
    case 1: hipLaunchKernelGGL((norm_row_kernel<Tag, 1, ALIGNED>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((norm_row_kernel<Tag, 2, ALIGNED>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((norm_row_kernel<Tag, 4, ALIGNED>), grid, block, 0, st, a); break;
    case 8: hipLaunchKernelGGL((norm_row_kernel<Tag, 8, ALIGNED>), grid, block, 0, st, a); break;
    default: return CAFEQ_ERR_UNSUPPORTED;
  }
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

bool rows_aligned(const void* p, int64_t ld, int size) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * size % 16 == 0);
}

int launch_rows(const RowArgs& a, int dtype, int64_t n, hipStream_t st) {
  const int size = dtype == CAFEQ_F32 ? 4 : 2;
  const bool al = a.d % kVec == 0 && rows_aligned(a.x, a.ldx, size) && rows_aligned(a.res, a.ldr, size) &&
                  rows_aligned(a.sum, a.lds, size) && rows_aligned(a.gain, 4, 4) &&
                  (reinterpret_cast<uintptr_t>(a.codes) & 7u) == 0 && rows_aligned(a.values, a.ldv, a.vdtype == CAFEQ_F32 ? 4 : 2);
  if (dtype == CAFEQ_F32) return al ? launch_rows_as<F32Tag, true>(a, n, st) : launch_rows_as<F32Tag, false>(a, n, st);
  return al ? launch_rows_as<BF16Tag, true>(a, n, st) : launch_rows_as<BF16Tag, false>(a, n, st);
}

// ---------------------------------------------------------------------------
// the transform
// ---------------------------------------------------------------------------
using bf16x8 = __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16;
using f32x16 = __attribute__((__vector_size__(16 * sizeof(float)))) float;

struct TileArgs {
  RowArgs r;             // r.group: 0 no codes, else a power of two that lies in a tile
  const float* Tinv;
  int64_t n;
};

union Frag { uint32_t u[4]; bf16x8 v; };

// eight float32 as three bfloat16 parts, hi + mid + lo exactly (8 + 8 + 8 significant bits, each part the leading bits of what
// the ones before it leave)
__device__ __forceinline__ void split3(const float (&x)[8], Frag& hi, Frag& mid, Frag& lo) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    uint32_t h[2], m[2], l[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float v = x[2 * p + e];
      h[e] = __float_as_uint(v) & 0xFFFF0000u;
      const float r1 = v - __uint_as_float(h[e]);
      m[e] = __float_as_uint(r1) & 0xFFFF0000u;
      l[e] = __float_as_uint(r1 - __uint_as_float(m[e]));
    }
    hi.u[p] = (h[0] >> 16) | h[1];
    mid.u[p] = (m[0] >> 16) | m[1];
    lo.u[p] = (l[0] >> 16) | (l[1] & 0xFFFF0000u);
  }
}

constexpr int kTok = 32;   // tokens a step

// A workgroup owns TC columns (whole blocks) and walks over tiles of 32 tokens.  z^T = Tinv y^T on the 16-bit matrix pipe with
// both operands in three bfloat16 parts and the six part products of weight >= 2^-24 (float32 accuracy: a code moves only where
// float32 arithmetic in another order moves it).  A wave holds its 32 rows of Tinv in registers for all its tiles; y passes
// through LDS, split once a workgroup.  In the accumulator a lane has 16 columns of ONE token, so that a group's maximum is a
// scan of registers, one exchange with lane ^ 32 and, for groups over 32, one through LDS.
// Bound: few tokens the launch and reading Tinv (64 KB a workgroup at blocks of 128), many the bytes of x, r and the outputs.
template <int K, class Tag>
__global__ __launch_bounds__(K == 256 ? 512 : 256) void act_tile_kernel(const TileArgs t) {
  constexpr int TC = K == 256 ? 256 : 128;
  constexpr int NW = TC / 32, NT = NW * 64;
  constexpr int STRIDE = TC + 8;                       // 16-bit elements: rows of 32 lanes fall on distinct banks in eights
  constexpr int KS = K / 16;
  constexpr int PER = kTok * TC / NT;                  // columns a thread stages: 16
  __shared__ uint16_t ys[3][kTok * STRIDE];
  __shared__ float zs[kTok * (TC + 4)];
  __shared__ uint32_t top[NW][kTok];
  const RowArgs& a = t.r;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
  const int64_t col0 = int64_t(blockIdx.x) * TC;       // the tile's first column
  const int64_t wcol = col0 + wave * 32;               // this wave's output columns
  const bool live = wcol < a.d;
  const int blk0 = wave * 32 / K * K;                  // first column of the wave's block inside the tile
  Frag ph[KS], pm[KS], pl[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (live) {
      const float* p = t.Tinv + (wcol + l32) * K + s * 16 + half * 8;   // row (wcol + l32) of the list of d rows of K floats
      const float4 u = *reinterpret_cast<const float4*>(p), v = *reinterpret_cast<const float4*>(p + 4);
      w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; w[4] = v.x; w[5] = v.y; w[6] = v.z; w[7] = v.w;
    }
    split3(w, ph[s], pm[s], pl[s]);
  }
  const int srow = tid * PER / TC, scol = tid * PER % TC;
  const int64_t ntile = (t.n + kTok - 1) / kTok;
  for (int64_t tile = blockIdx.y; tile < ntile; tile += gridDim.y) {
    const int64_t t0 = tile * kTok;
    // y of 32 tokens, split, into LDS
    {
      const int64_t row = t0 + srow, col = col0 + scol;
      const bool in = row < t.n && col < a.d;
      const float rstd = a.norm && in ? a.rstd[row] : 1.f;
#pragma unroll
      for (int c = 0; c < PER; c += 8) {
        float v[8];
        if (in) {
          load_vec<Tag, true>(v, a.x, row * a.ldx + col + c, 8);
          if (a.res) {
            float r[8];
            load_vec<Tag, true>(r, a.res, row * a.ldr + col + c, 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += r[e];
          }
          if (a.norm) {
            float g[8];
            if (a.gain) load_vec<F32Tag, true>(g, a.gain, col + c, 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = a.gain ? v[e] * rstd * (a.offset + g[e]) : v[e] * rstd;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = 0.f;
        }
        Frag h, m, l;
        split3(v, h, m, l);
        const int at = srow * STRIDE + scol + c;
        *reinterpret_cast<uint4*>(&ys[0][at]) = make_uint4(h.u[0], h.u[1], h.u[2], h.u[3]);
        *reinterpret_cast<uint4*>(&ys[1][at]) = make_uint4(m.u[0], m.u[1], m.u[2], m.u[3]);
        *reinterpret_cast<uint4*>(&ys[2][at]) = make_uint4(l.u[0], l.u[1], l.u[2], l.u[3]);
      }
    }
    __syncthreads();
    f32x16 acc = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      Frag yh, ym, yl;
      const int at = l32 * STRIDE + blk0 + s * 16 + half * 8;
      yh.v = *reinterpret_cast<const bf16x8*>(&ys[0][at]);
      ym.v = *reinterpret_cast<const bf16x8*>(&ys[1][at]);
      yl.v = *reinterpret_cast<const bf16x8*>(&ys[2][at]);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pm[s].v, ym.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pl[s].v, yh.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ph[s].v, yl.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pm[s].v, yh.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ph[s].v, ym.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ph[s].v, yh.v, acc, 0, 0, 0);
    }
    // register f of the lane: column 8 (f / 4) + 4 half + f % 4 of the wave's 32, token l32
    if (a.codes) {
      uint32_t m = 0u;
#pragma unroll
      for (int f = 0; f < 16; ++f) m = max(m, mag_bits(acc[f]));
      m = max(m, uint32_t(__shfl_xor(int(m), 32)));
      if (half == 0) top[wave][l32] = m;
    }
#pragma unroll
    for (int f = 0; f < 16; f += 4)
      *reinterpret_cast<float4*>(&zs[l32 * (TC + 4) + wave * 32 + 2 * f + 4 * half]) = make_float4(acc[f], acc[f + 1], acc[f + 2], acc[f + 3]);
    __syncthreads();
    // out, sixteen columns a thread
    const int64_t row = t0 + srow, col = col0 + scol;
    if (row < t.n && col < a.d) {
      float inv = 0.f, s = 0.f;
      if (a.codes) {
        uint32_t m = 0u;
        const int w0 = int(scol / a.group * a.group) / 32, w1 = w0 + int(a.group) / 32;
        for (int w = w0; w < w1; ++w) m = max(m, top[w][srow]);
        const float amax = __uint_as_float(m);
        inv = act_inv(amax);
        s = __fdiv_rn(amax, 127.f);
        if (scol % a.group == 0) a.scales[row * (a.d / a.group) + col / a.group] = s;
      }
#pragma unroll
      for (int c = 0; c < PER; c += 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          const float4 u = *reinterpret_cast<const float4*>(&zs[srow * (TC + 4) + scol + c + e]);
          v[e] = u.x; v[e + 1] = u.y; v[e + 2] = u.z; v[e + 3] = u.w;
        }
        if (a.codes) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = act_code(v[e], inv);
          *reinterpret_cast<uint2*>(a.codes + row * a.d + col + c) = make_uint2(pack4(v[0], v[1], v[2], v[3]), pack4(v[4], v[5], v[6], v[7]));
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], s);
        }
        if (a.values) store_vec<true>(v, a.values, a.vdtype, row * a.ldv + col + c, 8);
      }
    }
    __syncthreads();
  }
}

template <class Tag>
int launch_tiles(int k, const TileArgs& t, hipStream_t st) {
  const int tc = k == 256 ? 256 : 128;
  const int64_t cols = (t.r.d + tc - 1) / tc, ntile = (t.n + kTok - 1) / kTok;
  // four workgroups a compute unit: each splits its rows of Tinv once for the token tiles that it takes
  const int64_t want = (4 * device_cu_count() + cols - 1) / cols;
  const dim3 grid(unsigned(cols), unsigned(std::min<int64_t>(ntile, std::max<int64_t>(1, want))));
  switch (k) {
    case 32: hipLaunchKernelGGL((act_tile_kernel<32, Tag>), grid, dim3(256), 0, st, t); break;
    case 64: hipLaunchKernelGGL((act_tile_kernel<64, Tag>), grid, dim3(256), 0, st, t); break;
    case 128: hipLaunchKernelGGL((act_tile_kernel<128, Tag>), grid, dim3(256), 0, st, t); break;
    case 256: hipLaunchKernelGGL((act_tile_kernel<256, Tag>), grid, dim3(512), 0, st, t); break;
    default: return CAFEQ_ERR_UNSUPPORTED;
  }
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

// whether act_tile_kernel has all of a group in one tile
bool group_in_tile(int k, int64_t group) {
  const int64_t tc = k == 256 ? 256 : 128;
  return group <= tc && (group & (group - 1)) == 0;
}

bool overlaps(const void* a, int64_t bytes_a, const void* b, int64_t bytes_b) {
  const auto p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return a && b && p < q + uint64_t(bytes_b) && q < p + uint64_t(bytes_a);
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_norm_workspace_bytes(int64_t n, int64_t d, const cafeq_xform* xf, int64_t group) {
  if (n < 1 || d < 1 || !xf) return 0;
  const size_t rstd = align_up(size_t(n) * sizeof(float), 256);
  const bool whole = group >= 0 && !group_in_tile(xf->k, group == 0 ? d : group);
  return rstd + (whole ? align_up(size_t(n) * size_t(d) * sizeof(float), 256) : 0);
}

int cafeq_norm_quantize(const cafeq_activations* in, int64_t n, int64_t d, const cafeq_xform* xf, int64_t group,
                        int8_t* codes, float* scales, void* values, int values_dtype, int64_t ldv, void* ws,
                        void* stream) {
  if (!in || !in->x) return CAFEQ_ERR_INVALID_ARG;
  if (in->dtype != CAFEQ_F32 && in->dtype != CAFEQ_BF16) return CAFEQ_ERR_INVALID_ARG;
  if (values && values_dtype != CAFEQ_F32 && values_dtype != CAFEQ_BF16) return CAFEQ_ERR_INVALID_ARG;
  if ((codes == nullptr) != (scales == nullptr)) return CAFEQ_ERR_INVALID_ARG;
  if (!codes && !values) return CAFEQ_ERR_INVALID_ARG;
  if (n < 0 || d < 1 || in->ldx < d || (in->residual && in->ldr < d) || (in->sum && in->lds < d) || (values && ldv < d))
    return CAFEQ_ERR_BAD_SHAPE;
  if (d > kMaxRow || n > INT32_MAX) return CAFEQ_ERR_UNSUPPORTED;
  int64_t g = 0;
  if (codes) {
    if (group < 0 || (group > 0 && (group % kMinGroup != 0 || d % group != 0))) return CAFEQ_ERR_BAD_SHAPE;
    g = group == 0 ? d : group;
  }
  const int size = in->dtype == CAFEQ_F32 ? 4 : 2;
  auto aligned = [](const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; };
  if (!aligned(in->x, size) || !aligned(in->residual, size) || !aligned(in->sum, size) || !aligned(in->gain, 4) ||
      !aligned(scales, 4) || (values && !aligned(values, values_dtype == CAFEQ_F32 ? 4 : 2)))
    return CAFEQ_ERR_BAD_ALIGN;
  if (xf) {
    if (!xf->Tinv) return CAFEQ_ERR_INVALID_ARG;
    if (xf->k != 32 && xf->k != 64 && xf->k != 128 && xf->k != 256) return CAFEQ_ERR_UNSUPPORTED;
    if (xf->rep != 1 || int64_t(xf->nb) * xf->k != d) return CAFEQ_ERR_BAD_SHAPE;
    if (!aligned(xf->Tinv, 16) || !aligned(codes, 8) || !rows_aligned(in->x, in->ldx, size) ||
        !rows_aligned(in->residual, in->ldr, size) || !aligned(in->gain, 16) ||
        !rows_aligned(values, ldv, values_dtype == CAFEQ_F32 ? 4 : 2))
      return CAFEQ_ERR_BAD_ALIGN;
    if (!ws) return CAFEQ_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return CAFEQ_ERR_BAD_ALIGN;
    // x and residual are read a second time, after the sum has been written
    const int64_t span = size * ((n - 1) * in->lds + d);
    if (n > 0 && in->sum && (overlaps(in->sum, span, in->x, size * ((n - 1) * in->ldx + d)) ||
                             (in->residual && overlaps(in->sum, span, in->residual, size * ((n - 1) * in->ldr + d)))))
      return CAFEQ_ERR_INVALID_ARG;
  }
  if (n == 0) return CAFEQ_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  RowArgs a{};
  a.x = in->x; a.res = in->residual; a.sum = in->sum;
  a.ldx = in->ldx; a.ldr = in->ldr; a.lds = in->lds; a.d = d;
  a.gain = in->gain; a.offset = in->gain_offset; a.eps = in->eps; a.norm = in->norm;
  if (!xf) {
    a.group = g; a.codes = codes; a.scales = scales; a.values = values; a.ldv = ldv; a.vdtype = values_dtype;
    return launch_rows(a, in->dtype, n, st);
  }
  a.rstd = static_cast<float*>(ws);
  if (in->norm || in->sum) {
    const int rc = launch_rows(a, in->dtype, n, st);
    if (rc) return rc;
  }
  a.sum = nullptr;
  float* z = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(size_t(n) * sizeof(float), 256));
  const bool direct = !codes || group_in_tile(xf->k, g);
  TileArgs t{a, xf->Tinv, n};
  t.r.group = codes ? g : 0;
  if (direct) {
    t.r.codes = codes; t.r.scales = scales; t.r.values = values; t.r.ldv = ldv; t.r.vdtype = values_dtype;
  } else {
    t.r.values = z; t.r.ldv = d; t.r.vdtype = CAFEQ_F32;
  }
  int rc = in->dtype == CAFEQ_F32 ? launch_tiles<F32Tag>(xf->k, t, st) : launch_tiles<BF16Tag>(xf->k, t, st);
  if (rc || direct) return rc;
  // groups that no tile holds: z as it is, quantized row by row
  RowArgs q{};
  q.x = z; q.ldx = d; q.d = d; q.group = g; q.codes = codes; q.scales = scales; q.values = values; q.ldv = ldv; q.vdtype = values_dtype;
  return launch_rows(q, CAFEQ_F32, n, st);
}

}  // extern "C"
