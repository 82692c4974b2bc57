// Norm of each head of queries and keys, and their positions, in one pass:
//   y = x (mean x^2 + eps)^-1/2 (offset + gain),   (a, b) -> amplitude (a cos w - b sin w, a sin w + b cos w),   w = position * freq
// Bound by memory where there are many tokens and by the launch where there are few.
#include <math.h>

#include "cafeq_common.hpp"
#include "cafeq_internal.hpp"
#include "heads.hpp"

namespace cafeq {
namespace {

constexpr int kHeadMax = 512, kThreads = 256;

struct RotateArgs {
  cafeq_heads part[2];
  cafeq_rotation c;
  int64_t n;
  const int32_t* positions;
  const double* freq;
};

template <int LANES>
__device__ __forceinline__ float cluster_sum(float v) {
  if constexpr (LANES >= 2) v += dpp_mov<0xB1>(v);
  if constexpr (LANES >= 4) v += dpp_mov<0x4E>(v);
  if constexpr (LANES >= 8) v += dpp_mov<0x141>(v);
  if constexpr (LANES >= 16) v += dpp_mov<0x140>(v);
  if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
  if constexpr (LANES >= 64) v += __shfl_xor(v, 32);
  return v;
}

// N neighbouring elements at p + at as float32, and back
template <int N>
__device__ __forceinline__ void get(const float* p, float* v) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 f = load4(p + i);
      v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = p[i];
  }
}
template <int N>
__device__ __forceinline__ void get(const uint16_t* p, float* v) {
  uint32_t u[(N + 1) / 2];
  if constexpr (N == 8) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
  } else if constexpr (N == 4) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    u[0] = w.x; u[1] = w.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = bf16_bits_to_f32(p[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}
template <int N>
__device__ __forceinline__ void put(float* p, const float* v) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = v[i];
  }
}
template <int N>
__device__ __forceinline__ void put(uint16_t* p, const float* v) {
  if constexpr (N == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(bf16_bits(v[0], v[1]), bf16_bits(v[2], v[3]), bf16_bits(v[4], v[5]), bf16_bits(v[6], v[7]));
  } else if constexpr (N == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(bf16_bits(v[0], v[1]), bf16_bits(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = bf16_bits(v[i]);
  }
}

// A cluster of LANES lanes holds a head, each lane IT runs of VP pairs of channels: it forms the sines of its pairs once for the token and
// goes over the heads, NH of them requested at once.  Runs behind the turned ones are 2 VP neighbouring channels that stay.
// 4096 tokens of 16 and 8 heads of 256, bfloat16: 24.8 us (4.1 TB/s); with sines formed by every cluster 27.8.  One token of 48 heads: 3.3.
template <class Tag, int VP, int LANES, int IT, int NH>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
  using elem = typename Tag::elem;
  constexpr int kClusters = kThreads / LANES;
  const int lane = threadIdx.x % LANES, cluster = blockIdx.y * kClusters + threadIdx.x / LANES;
  const int step = gridDim.y * kClusters, heads = a.part[0].heads + a.part[1].heads;
  const int64_t t = blockIdx.x;
  const int half = a.c.rot / 2, turned = half / VP, runs = a.c.d / 2 / VP;
  int at[IT], gap[IT];     // first channel of a run, and how far the pairs' partners lie (0: 2 VP channels side by side)
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int r = lane + LANES * i;
    at[i] = r < turned && !a.c.interleaved ? r * VP : r * 2 * VP;
    gap[i] = r < turned && !a.c.interleaved ? half : 0;
  }
  float v[NH][IT][2 * VP];
  auto request = [&](int h0) {
#pragma unroll
    for (int k = 0; k < NH; ++k) {
      const int hh = h0 + k * step;
      const bool second = hh >= a.part[0].heads;
      const cafeq_heads& p = a.part[second];
      const elem* x = static_cast<const elem*>(p.x) + t * p.ldx + (second ? hh - a.part[0].heads : hh) * p.hsx;
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        if (hh < heads && lane + LANES * i < runs) {
          if (gap[i]) {
            get<VP>(x + at[i], v[k][i]);
            get<VP>(x + at[i] + gap[i], v[k][i] + VP);
          } else {
            get<2 * VP>(x + at[i], v[k][i]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 2 * VP; ++e) v[k][i][e] = 0.f;
        }
      }
    }
  };
  request(cluster);
  // The sines once for the workgroup.  Revolutions, whole ones taken off in float64; the rest, at most half, is
  // rounded to 24 bits (2^-25 of a revolution: 3.8e-8 on float32 results, against 2.9e-8 of an angle kept in float64); sincospi is good to float32's last bits of it, the
  // hardware's sine to 2^-20: 2^-12 of a step of bfloat16, and more only where a pair cancels
  __shared__ __align__(16) float cos_lds[kHeadMax / 2], sin_lds[kHeadMax / 2];
  if (threadIdx.x < half) {
    const double rev = a.positions[t] * 0.15915494309189533577 * a.freq[threadIdx.x];
    const float rest = float(rev - rint(rev));
    float s, c;
    if constexpr (Tag::dtype == CAFEQ_F32) {
      sincospif(2.f * rest, &s, &c);
    } else {
      s = __builtin_amdgcn_sinf(rest);
      c = __builtin_amdgcn_cosf(rest);
    }
    cos_lds[threadIdx.x] = c * a.c.amplitude;
    sin_lds[threadIdx.x] = s * a.c.amplitude;
  }
  __syncthreads();
  float cs[IT][VP], sn[IT][VP];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int r = lane + LANES * i;
    if (r >= turned) continue;
#pragma unroll
    for (int e = 0; e < VP; ++e) {
      cs[i][e] = cos_lds[r * VP + e];
      sn[i][e] = sin_lds[r * VP + e];
    }
  }
  for (int h0 = cluster; h0 < heads;) {
#pragma unroll
    for (int k = 0; k < NH; ++k) {
      const int hh = h0 + k * step;
      if (hh >= heads) continue;
      const bool second = hh >= a.part[0].heads;
      const cafeq_heads& p = a.part[second];
      elem* o = static_cast<elem*>(p.out) + t * p.ldo + (second ? hh - a.part[0].heads : hh) * p.hso;
      float scale = 1.f;
      if (a.c.norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int e = 0; e < 2 * VP; ++e) sum += v[k][i][e] * v[k][i][e];
        scale = 1.f / sqrtf(cluster_sum<LANES>(sum) / float(a.c.d) + a.c.eps);
      }
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        if (lane + LANES * i >= runs) continue;
        float(&x)[2 * VP] = v[k][i];
        if (a.c.norm) {
          float g[2 * VP];
          if (p.gain && gap[i]) {
            get<VP>(p.gain + at[i], g);
            get<VP>(p.gain + at[i] + gap[i], g + VP);
          } else if (p.gain) {
            get<2 * VP>(p.gain + at[i], g);
          }
#pragma unroll
          for (int e = 0; e < 2 * VP; ++e) x[e] = x[e] * scale * (p.gain ? a.c.gain_offset + g[e] : 1.f);
        }
        if (lane + LANES * i < turned) {
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            // the pair's places
            float &x0 = gap[i] ? x[e] : x[2 * e], &x1 = gap[i] ? x[VP + e] : x[2 * e + 1];
            const float y0 = x0, y1 = x1;
            x0 = y0 * cs[i][e] - y1 * sn[i][e];
            x1 = y0 * sn[i][e] + y1 * cs[i][e];
          }
        }
        if (gap[i]) {
          put<VP>(o + at[i], x);
          put<VP>(o + at[i] + gap[i], x + VP);
        } else {
          put<2 * VP>(o + at[i], x);
        }
      }
    }
    h0 += NH * step;
    if (h0 < heads) request(h0);
  }
}

template <class Tag, int VP, int LANES, int IT>
int launch(const RotateArgs& a, hipStream_t st) {
  const int heads = a.part[0].heads + a.part[1].heads, per = kThreads / LANES;
  // few tokens: the heads over several workgroups; many: one a token, whose sines serve all its heads
  const int y = a.n >= 256 ? 1 : (heads + per - 1) / per;
  hipLaunchKernelGGL((rotate_kernel<Tag, VP, LANES, IT, (IT > 1 ? 1 : 4)>), dim3(unsigned(a.n), unsigned(y)), dim3(kThreads), 0, st, a);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

template <class Tag>
int launch_type(const RotateArgs& a, bool wide, hipStream_t st) {
  if (!wide) return launch<Tag, 1, 64, kHeadMax / 128>(a, st);
  const int runs = a.c.d / 8;
  if (runs <= 8) return launch<Tag, 4, 8, 1>(a, st);
  if (runs <= 16) return launch<Tag, 4, 16, 1>(a, st);
  if (runs <= 32) return launch<Tag, 4, 32, 1>(a, st);
  return launch<Tag, 4, 64, 1>(a, st);
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

int cafeq_rotate_heads(const cafeq_rotation* cfg, const cafeq_heads* q, const cafeq_heads* k, int64_t n, const int32_t* positions,
                       const double* freq, void* stream) {
  if (!cfg || !positions || (!freq && cfg->rot) || (cfg->dtype != CAFEQ_F32 && cfg->dtype != CAFEQ_BF16)) return CAFEQ_ERR_INVALID_ARG;
  if (n < 0 || cfg->d < 2 || cfg->d % 2 || cfg->rot < 0 || cfg->rot % 2 || cfg->rot > cfg->d) return CAFEQ_ERR_BAD_SHAPE;
  if (cfg->d > kHeadMax || n > (int64_t(1) << 21)) return CAFEQ_ERR_UNSUPPORTED;
  RotateArgs a{{}, *cfg, n, positions, freq};
  const int size = cfg->dtype == CAFEQ_F32 ? 4 : 2;
  bool wide = cfg->d % 8 == 0 && cfg->rot % 8 == 0;
  const cafeq_heads* parts[2] = {q, k};
  HeadRows in[2] = {}, out[2] = {};
  for (int i = 0; i < 2; ++i) {
    if (!parts[i] || !parts[i]->x) continue;
    cafeq_heads& p = a.part[i] = *parts[i];
    if (!p.out) return CAFEQ_ERR_INVALID_ARG;
    if (p.heads < 1) return CAFEQ_ERR_BAD_SHAPE;
    if (p.heads > 4096) return CAFEQ_ERR_UNSUPPORTED;
    if (!aligned_to(p.x, size) || !aligned_to(p.out, size) || !aligned_to(p.gain, 4) || !aligned_to(positions, 4) || !aligned_to(freq, 8)) return CAFEQ_ERR_BAD_ALIGN;
    in[i] = {p.x, n, p.ldx, p.heads, p.hsx, cfg->d, size};
    out[i] = {p.out, n, p.ldo, p.heads, p.hso, cfg->d, size};
    if (p.ldx < 0 || p.hsx < 0 || !out[i].plain()) return CAFEQ_ERR_BAD_SHAPE;
    if (!in[i].same(out[i]) && may_share(in[i], out[i])) return CAFEQ_ERR_INVALID_ARG;
    wide = wide && aligned_to(p.x, 16) && aligned_to(p.out, 16) && aligned_to(p.gain, 16) && ((p.ldx | p.hsx | p.ldo | p.hso) & 7) == 0;
  }
  if (!a.part[0].heads && !a.part[1].heads) return CAFEQ_ERR_INVALID_ARG;
  // one part's output over the other's input, or over its output
  if (may_share(in[0], out[1]) || may_share(in[1], out[0]) || may_share(out[0], out[1])) return CAFEQ_ERR_INVALID_ARG;
  if (n == 0) return CAFEQ_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return cfg->dtype == CAFEQ_F32 ? launch_type<F32Tag>(a, wide, st) : launch_type<BF16Tag>(a, wide, st);
}

}  // extern "C"
