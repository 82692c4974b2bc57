// Activations of a quantized layer made ready in 8 bits: residual addition, root-mean-square norm, the blocks of the
// inverse transform (paper Sec. 4.1, the first factor of Y^ = X M^-1 Q(MW)) and a scale per group of columns.
//   h = x + r,  y = h (mean_c h_c^2 + eps)^-1/2 (offset + gain),  z_b = Tinv_b y_b,
//   a_G = max_{c in G} |z_c|,  q = rint(z fl(127 / a)),  s = a / 127.
// Without a transform one workgroup holds a row in registers and reads it once (norm_row_kernel).  With one, act_tile_kernel
// forms z: a block of z needs the whole row only through 1 / rms, which for many rows a launch of the row kernel leaves and for few
// every workgroup forms itself.
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
      for (int e = 0; e < 4; ++e) w[e] = bf16_bits(v[2 * e], v[2 * e + 1]);
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) if (e < left) p[e] = bf16_bits(v[e]);
    }
  }
}

// One workgroup a row, the row in registers: CH chunks of eight columns a thread.  Reads x and r once and writes each output
// once; bound by those bytes for long batches (4096 x 3584 in bfloat16 with sum, codes and values: 28.2 us, 4.7 TB/s, the rate of a large
// copy) and by the launch and one trip to memory for a few rows (2304 columns 3.4 us).
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
  RowArgs r;             // r.group: 0 no codes, else a power of two that lies in a tile; r.rstd null: the rows' norms formed here
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
    hi.u[p] = __builtin_amdgcn_perm(h[1], h[0], 0x07060302u);
    mid.u[p] = __builtin_amdgcn_perm(m[1], m[0], 0x07060302u);
    lo.u[p] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302u);
  }
}

// N consecutive elements (4 or 8) as loaded, and their stores
template <class Tag, int N> struct Raw;
template <int N> struct Raw<F32Tag, N> {
  float4 a[N / 4];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) a[i] = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at)[i];
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) { v[4 * i] = a[i].x; v[4 * i + 1] = a[i].y; v[4 * i + 2] = a[i].z; v[4 * i + 3] = a[i].w; }
  }
};
template <int N> struct Raw<BF16Tag, N> {
  uint32_t a[N / 2];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if constexpr (N == 8) {
      const uint4 u = *reinterpret_cast<const uint4*>(p);
      a[0] = u.x; a[1] = u.y; a[2] = u.z; a[3] = u.w;
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      a[0] = u.x; a[1] = u.y;
    }
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  }
};
template <int N>
__device__ __forceinline__ void store_cols(const float* v, void* base, int dtype, int64_t at) {
  if (dtype == CAFEQ_F32) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<float4*>(static_cast<float*>(base) + at + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = bf16_bits(v[2 * i], v[2 * i + 1]);
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}

// three parts (split3) of N values at columns `at` of the planes
template <int N, int PLANE>
__device__ __forceinline__ void put_parts(const float* v, uint16_t* ys, int at) {
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    // (the compiler keeps what the parts share)
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      uint32_t p[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float r = v[2 * i + e];
        for (int k = 0; k < part; ++k) r -= __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
        p[e] = __float_as_uint(r);
      }
      w[i] = __builtin_amdgcn_perm(p[1], p[0], 0x07060302u);
    }
    if constexpr (N == 8) *reinterpret_cast<uint4*>(ys + part * PLANE + at) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(ys + part * PLANE + at) = make_uint2(w[0], w[1]);
  }
}

constexpr int kTok = 32;        // tokens a step
constexpr int kFuseTok = 8;     // tokens whose norms every workgroup forms for itself
constexpr int kOut = 128;       // output columns of a workgroup

// Waves that share a block's contraction: few tokens (one tile) all that the longest chain of loads and products can be cut into, many
// as far as the rows of Tinv that a wave holds (12 registers for 16 of its columns) leave room for two (256) and four waves a SIMD.
constexpr int tile_split(int k, bool few) { return few ? (k >= 128 ? 4 : k == 64 ? 2 : 1) : (k >= 128 ? 2 : 1); }
constexpr int tile_waves(int k, bool few) { return few || k == 256 ? 2 : 4; }

// A workgroup owns 128 output columns and walks over tiles of 32 tokens.  z^T = Tinv y^T on the 16-bit matrix pipe with both
// operands in three bfloat16 parts and the six part products of weight >= 2^-24 (float32 accuracy: a code moves only where
// float32 arithmetic in another order moves it).  A wave holds 32 rows of Tinv and its share of their columns in registers for all
// its tiles; y passes through LDS, split once a workgroup, the next tile's x and r requested before this one's products; the waves'
// shares of z meet in LDS, in order.  In the accumulator a lane has 16 columns of ONE token.  Up to 8 tokens the workgroup forms the rows'
// norms itself: reading them costs it less than a launch.
// Bound: few tokens the launch and reading Tinv (64 KB a workgroup at blocks of 128; one token of 4608 columns 6.8 us, of 3584 through
// blocks of 256 9.3), many the vector instructions around the products (2048 x 4608, blocks of 128, sum, codes and values: 25 us after the 9 of
// the norms; groups that no tile holds, with z through memory and the row kernel after it, 10 us more).  Blocks of 64 of float32 rows, without their
// norms: four waves a SIMD spill 16 registers.
template <int K, int KW, class Tag, bool FUSED, int WAVES>
__global__ __launch_bounds__(256 * KW, WAVES) void act_tile_kernel(const TileArgs t) {
  constexpr int YC = K > kOut ? K : kOut;              // columns of y that the outputs need
  constexpr int NW = 4 * KW, NT = 64 * NW;
  constexpr int STRIDE = YC + 8;                       // 16-bit elements: rows of 32 lanes fall on distinct banks in eights
  constexpr int ZS = kOut + 4;
  constexpr int KS = K / 16 / KW;
  constexpr int PER = kTok * YC / NT, V = PER < 8 ? PER : 8, NC = PER / V;         // columns a thread stages,
  constexpr int OPER = kTok * kOut / NT, OV = OPER < 8 ? OPER : 8, ONC = OPER / OV;  // and puts out
  constexpr int PLANE = kTok * STRIDE;
  constexpr int ROOM = 3 * PLANE * 2 > KW * kTok * ZS * 4 ? 3 * PLANE * 2 : KW * kTok * ZS * 4;   // z takes the room of y
  static_assert(V >= 4 && OV >= 4, "sizes");
  __shared__ __align__(16) unsigned char room[ROOM];
  __shared__ __align__(16) float gs[YC];
  __shared__ float norms[kFuseTok][NW];                // sums of squares, by the waves of a row
  uint16_t* ys = reinterpret_cast<uint16_t*>(room);
  float* zs = reinterpret_cast<float*>(room);
  const RowArgs& a = t.r;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), cw = wave & 3, kw = wave >> 2;
  const int64_t col0 = int64_t(blockIdx.x) * kOut;     // first output column
  const int64_t ycol0 = col0 / YC * YC;                // first column of y
  const int64_t wcol = col0 + cw * 32;                 // this wave's output columns
  const bool live = wcol < a.d;
  const int in0 = (K > kOut ? 0 : cw * 32 / K * K) + kw * (K / KW);   // the wave's columns of y, inside the tile
  const int srow = tid * PER / YC, scol = tid * PER % YC;
  const int orow = tid * OPER / kOut, ocol = tid * OPER % kOut;
  const int64_t ycol = ycol0 + scol, ntile = (t.n + kTok - 1) / kTok;
  const bool mine = K <= kOut || (scol / kOut == int(blockIdx.x & 1));   // whose sums this workgroup writes

  Raw<Tag, V> rx[NC], rr[NC];
  float rstd = 1.f;
  // the places of this thread's columns, a tile's worth on after each
  const int64_t step = int64_t(gridDim.y) * kTok;
  int64_t row = int64_t(blockIdx.y) * kTok + srow, xat = row * a.ldx + ycol, rat = row * a.ldr + ycol, sat = row * a.lds + ycol;
  int64_t out = int64_t(blockIdx.y) * kTok + orow, cat = out * a.d + col0 + ocol, vat = out * a.ldv + col0 + ocol;
  const int gshift = a.codes ? __builtin_ctz(int(a.group)) : 0;            // a power of two
  const int64_t ngroup = a.d >> gshift;
  int64_t gat = out * ngroup + ((col0 + ocol) >> gshift);
  auto request = [&](int64_t at, int64_t x_at, int64_t r_at) __attribute__((always_inline)) {
    if (at < t.n && ycol < a.d) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        rx[c].load(a.x, x_at + V * c);
        if (a.res) rr[c].load(a.res, r_at + V * c);
      }
      if (!FUSED && a.norm) rstd = a.rstd[at];
    }
  };
  request(row, xat, rat);
  for (int c = tid; c < YC; c += NT) gs[c] = a.norm && a.gain && ycol0 + c < a.d ? a.offset + a.gain[ycol0 + c] : 1.f;
  Frag ph[KS], pm[KS], pl[KS];
  int per = 1;                                         // (fused) waves of a row
  {
    float4 w[KS][2];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const float* p = t.Tinv + (wcol + l32) * K + kw * (K / KW) + s * 16 + half * 8;   // row (wcol + l32) of the list of d rows of K floats
      w[s][0] = live ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
      w[s][1] = live ? *reinterpret_cast<const float4*>(p + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if constexpr (FUSED) {
      // (blockIdx.y has one value then: all tokens are in the first tile.)  Waves that have no row of their own share one
      const int n = int(t.n);
      while (per * 2 * n <= NW) per *= 2;
      constexpr int ROWS = kFuseTok / NW > 0 ? kFuseTok / NW : 1, FLY = Tag::dtype == CAFEQ_F32 ? 2 : 4;   // rows of a wave; requests of each under way
      const int first = wave % per * 512 + lane * 8;
      float sum[ROWS] = {};
      for (int64_t at0 = first; at0 < a.d; at0 += per * 512 * FLY) {
        Raw<Tag, 8> u[ROWS][FLY], q[ROWS][FLY];
#pragma unroll
        for (int i = 0; i < FLY; ++i)
#pragma unroll
          for (int r = 0; r < ROWS; ++r) {
            const int64_t at = at0 + i * per * 512;
            const int row = wave / per + r * (NW / per);
            if (row < n && at < a.d) {
              u[r][i].load(a.x, row * a.ldx + at);
              if (a.res) q[r][i].load(a.res, row * a.ldr + at);
            }
          }
#pragma unroll
        for (int i = 0; i < FLY; ++i)
#pragma unroll
          for (int r = 0; r < ROWS; ++r)
            if (wave / per + r * (NW / per) < n && at0 + i * per * 512 < a.d) {
              float v[8], z[8];
              u[r][i].get(v);
              if (a.res) q[r][i].get(z);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                if (a.res) v[e] += z[e];
                sum[r] = fmaf(v[e], v[e], sum[r]);
              }
            }
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int row = wave / per + r * (NW / per);
        const float s = wave_sum(sum[r]);
        if (lane == 0 && row < n) norms[row][wave % per] = s;
      }
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const float v[8] = {w[s][0].x, w[s][0].y, w[s][0].z, w[s][0].w, w[s][1].x, w[s][1].y, w[s][1].z, w[s][1].w};
      split3(v, ph[s], pm[s], pl[s]);
    }
  }
  __syncthreads();
  for (int64_t tile = blockIdx.y; tile < ntile; tile += gridDim.y) {
    {
      const bool in = row < t.n && ycol < a.d;
      if (FUSED && in) {
        float s = norms[srow][0];
        for (int w = 1; w < per; ++w) s += norms[srow][w];
        rstd = 1.f / sqrtf(s / float(a.d) + a.eps);
      }
      // y of 32 tokens, split, into LDS
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float v[V];
        if (in) {
          rx[c].get(v);
          if (a.res) {
            float r[V];
            rr[c].get(r);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += r[e];
          }
          if (a.sum && mine) store_cols<V>(v, a.sum, Tag::dtype, sat + V * c);
          if (a.norm) {
#pragma unroll
            for (int e = 0; e < V; e += 4) {
              const float4 g = *reinterpret_cast<const float4*>(&gs[scol + V * c + e]);
              v[e] = v[e] * rstd * g.x; v[e + 1] = v[e + 1] * rstd * g.y; v[e + 2] = v[e + 2] * rstd * g.z; v[e + 3] = v[e + 3] * rstd * g.w;
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) v[e] = 0.f;
        }
        put_parts<V, PLANE>(v, ys, srow * STRIDE + scol + V * c);
      }
    }
    __syncthreads();
    row += step; xat += step * a.ldx; rat += step * a.ldr; sat += step * a.lds;
    if (tile + gridDim.y < ntile) request(row, xat, rat);
    f32x16 acc = {};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      Frag yh, ym, yl;
      const int at = l32 * STRIDE + in0 + s * 16 + half * 8;
      yh.v = *reinterpret_cast<const bf16x8*>(ys + at);
      ym.v = *reinterpret_cast<const bf16x8*>(ys + PLANE + at);
      yl.v = *reinterpret_cast<const bf16x8*>(ys + 2 * PLANE + at);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pm[s].v, ym.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pl[s].v, yh.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ph[s].v, yl.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pm[s].v, yh.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ph[s].v, ym.v, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ph[s].v, yh.v, acc, 0, 0, 0);
    }
    __syncthreads();                                   // y has been read: z takes its room
    // register f of the lane: column 8 (f / 4) + 4 half + f % 4 of the wave's 32, token l32
#pragma unroll
    for (int f = 0; f < 16; f += 4)
      *reinterpret_cast<float4*>(&zs[(kw * kTok + l32) * ZS + cw * 32 + 2 * f + 4 * half]) = make_float4(acc[f], acc[f + 1], acc[f + 2], acc[f + 3]);
    __syncthreads();
    // out; a thread's columns lie in one run of 32, and so in one group
    const bool in = out < t.n && col0 + ocol < a.d;
    float v[OPER];
#pragma unroll
    for (int e = 0; e < OPER; e += 4) {
      float4 u = *reinterpret_cast<const float4*>(&zs[orow * ZS + ocol + e]);
#pragma unroll
      for (int k = 1; k < KW; ++k) {
        const float4 w = *reinterpret_cast<const float4*>(&zs[(k * kTok + orow) * ZS + ocol + e]);
        u.x += w.x; u.y += w.y; u.z += w.z; u.w += w.w;
      }
      v[e] = u.x; v[e + 1] = u.y; v[e + 2] = u.z; v[e + 3] = u.w;
    }
    if (a.codes) {
      // a group is g / OPER neighbouring threads (OPER divides 32): at most 32 lanes of a wave
      const int g = 1 << gshift;
      uint32_t m = 0u;
#pragma unroll
      for (int e = 0; e < OPER; ++e) m = max(m, mag_bits(v[e]));
      m = cluster_umax(m, g / OPER);
      const float amax = __uint_as_float(m), inv = act_inv(amax), s = __fdiv_rn(amax, 127.f);
      if (in && (ocol & (g - 1)) == 0) a.scales[gat] = s;
      uint32_t q[OPER / 4];
#pragma unroll
      for (int e = 0; e < OPER; ++e) v[e] = act_code(v[e], inv);
#pragma unroll
      for (int e = 0; e < OPER / 4; ++e) q[e] = pack4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
      if (in) {
        int8_t* p = a.codes + cat;
        if constexpr (OPER == 16) *reinterpret_cast<uint4*>(p) = make_uint4(q[0], q[1], q[2], q[3]);
        else if constexpr (OPER == 8) *reinterpret_cast<uint2*>(p) = make_uint2(q[0], q[1]);
        else *reinterpret_cast<uint32_t*>(p) = q[0];
      }
#pragma unroll
      for (int e = 0; e < OPER; ++e) v[e] = __fmul_rn(v[e], s);
    }
    if (a.values && in)
#pragma unroll
      for (int c = 0; c < ONC; ++c) store_cols<OV>(v + OV * c, a.values, a.vdtype, vat + OV * c);
    out += step; cat += step * a.d; vat += step * a.ldv; gat += step * ngroup;
    __syncthreads();
  }
}

template <class Tag, int K>
int launch_tile_k(const TileArgs& t, hipStream_t st) {
  const int64_t cols = (t.r.d + kOut - 1) / kOut, ntile = (t.n + kTok - 1) / kTok;
  constexpr int KF = tile_split(K, true), KM = tile_split(K, false);
  if (ntile == 1) {
    const dim3 grid{unsigned(cols)}, block(256 * KF);
    if (t.r.norm && !t.r.rstd) hipLaunchKernelGGL((act_tile_kernel<K, KF, Tag, true, tile_waves(K, true)>), grid, block, 0, st, t);
    else hipLaunchKernelGGL((act_tile_kernel<K, KF, Tag, false, tile_waves(K, true)>), grid, block, 0, st, t);
  } else {
    // what fits the chip at once: each workgroup splits its rows of Tinv once for the token tiles that it takes
    const int64_t want = std::max<int64_t>(1, tile_waves(K, false) / KM * device_cu_count() / cols);
    const dim3 grid(unsigned(cols), unsigned(std::min<int64_t>(ntile, want)));
    hipLaunchKernelGGL((act_tile_kernel<K, KM, Tag, false, tile_waves(K, false)>), grid, dim3(256 * KM), 0, st, t);
  }
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

template <class Tag>
int launch_tiles(int k, const TileArgs& t, hipStream_t st) {
  switch (k) {
    case 32: return launch_tile_k<Tag, 32>(t, st);
    case 64: return launch_tile_k<Tag, 64>(t, st);
    case 128: return launch_tile_k<Tag, 128>(t, st);
    case 256: return launch_tile_k<Tag, 256>(t, st);
    default: return CAFEQ_ERR_UNSUPPORTED;
  }
}

// whether act_tile_kernel has all of a group in one tile
bool group_in_tile(int64_t group) { return group <= kOut && (group & (group - 1)) == 0; }

// 1 / rms of the rows, where a launch of its own forms them
size_t norms_bytes(int64_t n) { return n > kFuseTok ? align_up(size_t(n) * sizeof(float), 256) : 0; }

// Whether rows of d elements at a (leading dimension lda) and at b share memory.  Of rows with one leading dimension only their columns decide:
// slices side by side of one buffer do not overlap.
bool overlaps(const void* a, int64_t lda, const void* b, int64_t ldb, int64_t n, int64_t d, int size) {
  if (!a || !b || n < 1) return false;
  const auto p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  const uint64_t row = uint64_t(d) * size, sa = uint64_t(n - 1) * lda * size + row, sb = uint64_t(n - 1) * ldb * size + row;
  if (p >= q + sb || q >= p + sa) return false;
  if (n == 1 || lda != ldb) return true;
  const uint64_t ld = uint64_t(lda) * size, off = (p > q ? p - q : q - p) % ld;
  return off < row || off > ld - row;
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_norm_workspace_bytes(int64_t n, int64_t d, const cafeq_xform* xf, int64_t group) {
  if (n < 1 || d < 1 || !xf) return 0;
  const bool whole = group >= 0 && !group_in_tile(group == 0 ? d : group);
  return norms_bytes(n) + (whole ? align_up(size_t(n) * size_t(d) * sizeof(float), 256) : 0);
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
  cafeq_activations single;
  if (n == 1) {   // a single row has no next one: as if it lay alone
    single = *in;
    single.ldx = single.ldr = single.lds = ldv = d;
    in = &single;
  }
  if (d > kMaxRow || n > (int64_t(1) << 21)) return CAFEQ_ERR_UNSUPPORTED;   // a launch's threads stay below 2^32
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
    if (!aligned(xf->Tinv, 16) || !rows_aligned(in->x, in->ldx, size) ||
        !rows_aligned(in->residual, in->ldr, size) || !rows_aligned(in->sum, in->lds, size) || !aligned(codes, 16) ||
        !rows_aligned(values, ldv, values_dtype == CAFEQ_F32 ? 4 : 2))
      return CAFEQ_ERR_BAD_ALIGN;
    if (!ws && cafeq_norm_workspace_bytes(n, d, xf, codes ? group : -1)) return CAFEQ_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return CAFEQ_ERR_BAD_ALIGN;
  }
  // the sum's elements may take the place of those that they come from, where nothing reads these again; no other overlap
  auto bad_sum = [&](const void* from, int64_t ld) {
    if (!xf && in->sum == from && in->lds == ld) return false;
    return overlaps(in->sum, in->lds, from, ld, n, d, size);
  };
  if (in->sum && (bad_sum(in->x, in->ldx) || bad_sum(in->residual, in->ldr))) return CAFEQ_ERR_INVALID_ARG;
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
  if (in->norm && norms_bytes(n)) {
    a.rstd = static_cast<float*>(ws);
    RowArgs norms = a;
    norms.sum = nullptr;                      // written where z is formed
    const int rc = launch_rows(norms, in->dtype, n, st);
    if (rc) return rc;
  }
  float* z = reinterpret_cast<float*>(static_cast<char*>(ws) + norms_bytes(n));
  const bool direct = !codes || group_in_tile(g);
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
