// The cache of keys and values in 8 bits: storing new tokens, reading back what the codes stand for.
#include "cache.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kThreads = 256;

struct AppendArgs {
  cafeq_cache c;
  const void* x[2];         // keys, values
  int64_t ld[2], hs[2];
  const int32_t* starts;
  int n;
  int longest;
  Units units;
};

__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ void get8(const float* p, float* v) {
  const float4 a = load4(p), b = load4(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void get8(const uint16_t* p, float* v) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ float code_of(float x, float inv) { return fminf(fmaxf(__builtin_rintf(__fmul_rn(x, inv)), -127.f), 127.f); }
// four earlier codes on a larger scale; those from `keep` on stay
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float ratio, int keep) {
  uint32_t r = 0;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int q = int(w << (24 - 8 * b)) >> 24;
    const int z = b < keep ? int(__builtin_rintf(__fmul_rn(float(q), ratio))) : q;
    r |= (uint32_t(z) & 0xFFu) << (8 * b);
  }
  return r;
}

// A workgroup stores what a sequence's new tokens bring to one page and head, keys or values.
template <class Tag>
__global__ __launch_bounds__(kThreads) void append_kernel(const AppendArgs a) {
  using elem = typename Tag::elem;
  __shared__ uint32_t top[kThreads / 64];
  const cafeq_cache& c = a.c;
  const int head = blockIdx.y, side = blockIdx.z, tid = threadIdx.x, B = c.block, d = c.d;
  const int64_t w = blockIdx.x;
  const int i = sequence_of(a.units, a.starts, c.sequences, a.n, w);
  if (i < 0) return;
  const RowRange r = rows_of(a.starts, i, a.n);
  const int len = tokens_of(c, i), pos0 = len - (r.hi - r.lo);                 // row lo + j stands at pos0 + j
  const int64_t block = max(pos0, 0) / B + (w - a.units.base(r.lo, i));
  const int64_t first = max(int64_t(pos0), block * B);
  const int64_t last = min(min(int64_t(len), int64_t(pos0) + a.longest), (block + 1) * B);
  if (first >= last) return;
  const int page = page_of(c, i, int(block));
  if (page < 0) return;
  const int f = int(first - block * B), m = int(last - first), per = d / 8;
  const elem* x = static_cast<const elem*>(a.x[side]) + (r.lo + first - pos0) * a.ld[side] + head * a.hs[side];
  const int64_t at = int64_t(page) * c.heads + head;
  int8_t* codes = (side ? c.v : c.k) + at * B * d;
  float* scale = (side ? c.vscale : c.kscale) + at;

  uint32_t big = 0;
  for (int e = tid; e < m * per; e += kThreads) {
    float v[8];
    get8(x + (e / per) * a.ld[side] + e % per * 8, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) big = max(big, mag(v[j]));
  }
  for (int s = 1; s < 64; s <<= 1) big = max(big, uint32_t(__shfl_xor(int(big), s)));
  if ((tid & 63) == 0) top[tid >> 6] = big;
  const float old = f > 0 ? __uint_as_float(mag(*scale)) : 0.f;
  __syncthreads();
  for (int j = 0; j < kThreads / 64; ++j) big = max(big, top[j]);
  // compared as bits: a NaN lies above an infinity, and that above all numbers
  const float s = __uint_as_float(max(mag(old), mag(__fdiv_rn(__uint_as_float(big), 127.f))));
  const bool number = mag(s) < 0x7F800000u;
  const float inv = number && s > 0.f ? fminf(__fdiv_rn(1.f, s), FLT_MAX) : 0.f;
  if (f > 0 && mag(s) != mag(old)) {
    const float ratio = number ? __fdiv_rn(old, s) : 0.f;
    if (side == 0) {
      for (int e = tid; e < f * d / 4; e += kThreads) {
        uint32_t* p = reinterpret_cast<uint32_t*>(codes) + e;
        *p = rescaled(*p, ratio, 4);
      }
    } else {
      const int words = (f + 3) / 4;
      for (int e = tid; e < d * words; e += kThreads) {
        uint32_t* p = reinterpret_cast<uint32_t*>(codes + e / words * B) + e % words;
        *p = rescaled(*p, ratio, min(4, f - 4 * (e % words)));
      }
    }
  }
  if (tid == 0) *scale = s;
  __syncthreads();      // a word of v may hold earlier and new tokens
  for (int e = tid; e < m * per; e += kThreads) {
    const int t = e / per, ch = e % per * 8;
    float v[8];
    get8(x + t * a.ld[side] + ch, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = number ? code_of(v[j], inv) : 0.f;
    if (side == 0) {
      *reinterpret_cast<uint2*>(codes + (f + t) * d + ch) = make_uint2(pack4(v[0], v[1], v[2], v[3]), pack4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) codes[(ch + j) * B + f + t] = int8_t(int(v[j]));
    }
  }
}

struct ValueArgs {
  cafeq_cache c;
  const int32_t *begin, *starts;
  int n;
  void* out[2];
  Units units;
};

template <class Tag>
__global__ __launch_bounds__(kThreads) void values_kernel(const ValueArgs a) {
  using elem = typename Tag::elem;
  const cafeq_cache& c = a.c;
  const int head = blockIdx.y, side = blockIdx.z, tid = threadIdx.x, B = c.block, d = c.d;
  if (!a.out[side]) return;
  const int64_t w = blockIdx.x;
  const int i = sequence_of(a.units, a.starts, c.sequences, a.n, w);
  if (i < 0) return;
  const RowRange r = rows_of(a.starts, i, a.n);
  const int64_t pos0 = a.begin[i], rows = r.hi - r.lo, len = tokens_of(c, i);
  // blocks of positions, counted from the one that holds begin (negative positions included)
  const int64_t block = (pos0 >= 0 ? pos0 / B : -((-pos0 + B - 1) / B)) + (w - a.units.base(r.lo, i));
  const int64_t first = max(pos0, block * B), last = min(pos0 + rows, (block + 1) * B);
  if (first >= last) return;
  const int page = first >= 0 && first < len ? page_of(c, i, int(block)) : -1;
  const int64_t at = int64_t(max(page, 0)) * c.heads + head;
  const int8_t* codes = (side ? c.v : c.k) + at * B * d;
  const float s = page < 0 ? 0.f : (side ? c.vscale : c.kscale)[at];
  elem* out = static_cast<elem*>(a.out[side]) + ((r.lo + first - pos0) * c.heads + head) * d;
  const int f = int(first - block * B), m = int(last - first), per = d / 8;
  for (int e = tid; e < m * per; e += kThreads) {
    const int t = side ? e % m : e / per, ch = side ? e / m * 8 : e % per * 8;
    const bool there = page >= 0 && first + t < len;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = there ? __fmul_rn(float(side ? codes[(ch + j) * B + f + t] : codes[(f + t) * d + ch + j]), s) : 0.f;
    elem* o = out + int64_t(t) * c.heads * d + ch;
    if constexpr (Tag::dtype == CAFEQ_F32) {
      reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(o) = make_uint4(bf16_bits(v[0], v[1]), bf16_bits(v[2], v[3]), bf16_bits(v[4], v[5]), bf16_bits(v[6], v[7]));
    }
  }
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

int cafeq_cache_append(const cafeq_cache* cache, const void* k, const void* v, int dtype, int64_t n, int64_t ldk, int64_t hsk,
                       int64_t ldv, int64_t hsv, const int32_t* starts, int64_t longest, void* stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (!k || !v || !starts || (dtype != CAFEQ_F32 && dtype != CAFEQ_BF16)) return CAFEQ_ERR_INVALID_ARG;
  if (n < 0 || longest < 0 || ldk < 0 || hsk < 0 || ldv < 0 || hsv < 0) return CAFEQ_ERR_BAD_SHAPE;
  if (n > (int64_t(1) << 24)) return CAFEQ_ERR_UNSUPPORTED;
  const int per16 = dtype == CAFEQ_F32 ? 4 : 8;
  if (!aligned_to(k, 16) || !aligned_to(v, 16) || (ldk | hsk | ldv | hsv) % per16 || !aligned_to(starts, 4)) return CAFEQ_ERR_BAD_ALIGN;
  if (n == 0 || longest == 0 || cache->sequences == 0) return CAFEQ_OK;
  longest = std::min(longest, n);
  // a sequence's tokens touch at most floor of their number over the block, plus 2, pages; one token a sequence: one
  const Units u = longest == 1 ? Units{0, 1, 1} : Units{1, cache->block, 2};
  const AppendArgs a{*cache, {k, v}, {ldk, ldv}, {hsk, hsv}, starts, int(n), int(longest), u};
  const dim3 grid(unsigned(u.count(n, cache->sequences)), unsigned(cache->heads), 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == CAFEQ_F32) hipLaunchKernelGGL((append_kernel<F32Tag>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((append_kernel<BF16Tag>), grid, dim3(kThreads), 0, st, a);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

int cafeq_cache_values(const cafeq_cache* cache, const int32_t* begin, const int32_t* starts, int64_t n, void* k, void* v, int dtype,
                       void* stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (!begin || !starts || (!k && !v) || (dtype != CAFEQ_F32 && dtype != CAFEQ_BF16)) return CAFEQ_ERR_INVALID_ARG;
  if (n < 0) return CAFEQ_ERR_BAD_SHAPE;
  if (n > (int64_t(1) << 24)) return CAFEQ_ERR_UNSUPPORTED;
  if (!aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(begin, 4) || !aligned_to(starts, 4)) return CAFEQ_ERR_BAD_ALIGN;
  if (n == 0 || cache->sequences == 0) return CAFEQ_OK;
  const Units u{1, cache->block, 2};
  const ValueArgs a{*cache, begin, starts, int(n), {k, v}, u};
  const dim3 grid(unsigned(u.count(n, cache->sequences)), unsigned(cache->heads), 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == CAFEQ_F32) hipLaunchKernelGGL((values_kernel<F32Tag>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((values_kernel<BF16Tag>), grid, dim3(kThreads), 0, st, a);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

}  // extern "C"
