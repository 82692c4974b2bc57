// The cache of keys and values in 8 bits: storing new tokens, reading back what the codes stand for.
#include "cache.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kThreads = 256, kFewThreads = 64;

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

__device__ __forceinline__ uint4 rescaled(const uint4& w, float ratio, int keep) {
  return make_uint4(rescaled(w.x, ratio, keep), rescaled(w.y, ratio, keep - 4), rescaled(w.z, ratio, keep - 8), rescaled(w.w, ratio, keep - 12));
}

// A workgroup stores what a sequence's new tokens bring to one page and head, keys or values.  A thread takes eight channels of four tokens that
// share a dword of v, reads them once, and writes them as eight codes a token (k) or four a channel (v).  NG: such groups a thread holds.
// Bound by memory, and for single tokens by five loads one after another (starts, length, page, token, scale).  8192 tokens of 8 heads of 256: 30 us (3.4 TB/s; read
// twice, with v stored byte by byte, 82); one token each of 64 sequences, 16 heads of 128: 8.2.
template <class Tag, int T, int NG>
__global__ __launch_bounds__(T) void append_kernel(const AppendArgs a) {
  using elem = typename Tag::elem;
  __shared__ uint32_t top[T / 64];
  const cafeq_cache& c = a.c;
  const int head = blockIdx.y, side = blockIdx.z, tid = threadIdx.x, B = c.block, d = c.d;
  const int64_t w = blockIdx.x;
  const int i = a.longest == 1 ? int(w) : sequence_of(a.units, a.starts, c.sequences, a.n, w);
  if (i < 0) return;
  const bool closed = no_room(c, a.starts);
  const RowRange r = rows_of(a.starts, i, a.n);
  const int len = tokens_of(c, i), pos0 = len - (r.hi - r.lo);                 // row lo + j stands at pos0 + j
  const int64_t block = max(pos0, 0) / B + (w - a.units.base(r.lo, i));
  const int64_t first = max(int64_t(pos0), block * B);
  const int64_t last = min(min(int64_t(len), int64_t(pos0) + a.longest), (block + 1) * B);
  if (first >= last || closed) return;
  const int page = page_of(c, i, int(block));
  if (page < 0) return;
  const int f = int(first - block * B), m = int(last - first), per = d / 8;
  const int64_t ld = a.ld[side];
  // row of slot 0 of the page
  const elem* x = static_cast<const elem*>(a.x[side]) + (r.lo + block * B - pos0) * ld + head * a.hs[side];
  const int64_t at = int64_t(page) * c.heads + head;
  int8_t* codes = (side ? c.v : c.k) + at * B * d;
  float* scale = (side ? c.vscale : c.kscale) + at;

  const int group0 = f >> 2, groups = ((f + m - 1) >> 2) - group0 + 1, total = groups * per;
  float v[NG][4][8];
  uint32_t big = 0;
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    const int e = tid + n * T, ch = (side ? e / groups : e % per) * 8, slot = 4 * (group0 + (side ? e % groups : e / per));
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (e < total && slot + s >= f && slot + s < f + m) {
        get8(x + (slot + s) * ld + ch, v[n][s]);
#pragma unroll
        for (int j = 0; j < 8; ++j) big = max(big, mag(v[n][s][j]));
      }
  }
  const float old = f > 0 ? __uint_as_float(mag(*scale)) : 0.f;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) big = max(big, uint32_t(__shfl_xor(int(big), s)));
  if constexpr (T > 64) {
    if ((tid & 63) == 0) top[tid >> 6] = big;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T / 64; ++j) big = max(big, top[j]);
  }
  // compared as bits: a NaN lies above an infinity, and that above all numbers
  const float s = __uint_as_float(max(mag(old), mag(__fdiv_rn(__uint_as_float(big), 127.f))));
  const bool number = mag(s) < 0x7F800000u;
  const float inv = number && s > 0.f ? fminf(__fdiv_rn(1.f, s), FLT_MAX) : 0.f;
  if (f > 0 && mag(s) != mag(old)) {
    const float ratio = number ? __fdiv_rn(old, s) : 0.f;
    const int runs = side ? (f + 15) / 16 : d / 16, count = side ? d * runs : f * runs;
    for (int e = tid; e < count; e += T) {
      uint4* p = reinterpret_cast<uint4*>(codes + (side ? e / runs * B : e / runs * d)) + e % runs;
      *p = rescaled(*p, ratio, side ? f - 16 * (e % runs) : 16);
    }
    __syncthreads();      // a word of v may hold earlier and new tokens
  }
  if (tid == 0) *scale = s;
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    const int e = tid + n * T, ch = (side ? e / groups : e % per) * 8, slot = 4 * (group0 + (side ? e % groups : e / per));
    if (e >= total) continue;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[n][q][j] = number ? code_of(v[n][q][j], inv) : 0.f;
    const int lo = f - slot, hi = f + m - slot;      // of the four tokens
    if (side == 0) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q >= lo && q < hi)
          *reinterpret_cast<uint2*>(codes + (slot + q) * d + ch) =
              make_uint2(pack4(v[n][q][0], v[n][q][1], v[n][q][2], v[n][q][3]), pack4(v[n][q][4], v[n][q][5], v[n][q][6], v[n][q][7]));
    } else if (lo <= 0 && hi >= 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) *reinterpret_cast<uint32_t*>(codes + (ch + j) * B + slot) = pack4(v[n][0][j], v[n][1][j], v[n][2][j], v[n][3][j]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q >= lo && q < hi) {
#pragma unroll
          for (int j = 0; j < 8; ++j) codes[(ch + j) * B + slot + q] = int8_t(int(v[n][q][j]));
        }
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

// Slots f .. f + m - 1 of a page and head; row0: the row of slot 0; slots from `known` on, and those of a page that is not there, are zeros
template <class Tag>
__device__ __forceinline__ void page_values(const ValueArgs& a, int side, int head, int page, int64_t row0, int f, int m, int known) {
  using elem = typename Tag::elem;
  const cafeq_cache& c = a.c;
  const int tid = threadIdx.x, B = c.block, d = c.d, per = d / 8;
  const int64_t at = int64_t(max(page, 0)) * c.heads + head;
  const int8_t* codes = (side ? c.v : c.k) + at * B * d;
  const float s = page < 0 ? 0.f : (side ? c.vscale : c.kscale)[at];
  elem* out = static_cast<elem*>(a.out[side]) + (row0 * c.heads + head) * d;
  const int64_t ld = int64_t(c.heads) * d;
  auto store = [&](int slot, int ch, const float* v) {
    elem* o = out + slot * ld + ch;
    if constexpr (Tag::dtype == CAFEQ_F32) {
      reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(o) = make_uint4(bf16_bits(v[0], v[1]), bf16_bits(v[2], v[3]), bf16_bits(v[4], v[5]), bf16_bits(v[6], v[7]));
    }
  };
  if (side == 0) {
    for (int e = tid; e < m * per; e += kThreads) {
      const int slot = f + e / per, ch = e % per * 8;
      float v[8];
      const uint2 q = slot < known ? *reinterpret_cast<const uint2*>(codes + slot * d + ch) : make_uint2(0u, 0u);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(float(int8_t((j < 4 ? q.x : q.y) >> (8 * (j & 3)))), slot < known ? s : 0.f);
      store(slot, ch, v);
    }
    return;
  }
  // eight channels of four tokens that share a dword
  const int group0 = f >> 2, groups = ((f + m - 1) >> 2) - group0 + 1;
  for (int e = tid; e < groups * per; e += kThreads) {
    const int slot = 4 * (group0 + e % groups), ch = e / groups * 8;
    uint32_t q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = page < 0 ? 0u : *reinterpret_cast<const uint32_t*>(codes + (ch + j) * B + slot);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (slot + k < f || slot + k >= f + m) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = slot + k < known ? __fmul_rn(float(int8_t(q[j] >> (8 * k))), s) : 0.f;
      store(slot + k, ch, v);
    }
  }
}

// A workgroup: what one page and head hold of a sequence's rows, keys or values.  8192 tokens of 8 heads of 256 to bfloat16: 20 us (5.0 TB/s); four heads a
// workgroup 24.
template <class Tag>
__global__ __launch_bounds__(kThreads) void values_kernel(const ValueArgs a) {
  const cafeq_cache& c = a.c;
  const int side = blockIdx.z, B = c.block;
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
  page_values<Tag>(a, side, int(blockIdx.y), page, r.lo + block * B - pos0, int(first - block * B), int(last - first),
                   page < 0 ? 0 : int(min(int64_t(B), len - block * B)));
}

template <class Tag>
int launch_append(const AppendArgs& a, hipStream_t st) {
  const dim3 grid(unsigned(a.units.count(a.n, a.c.sequences)), unsigned(a.c.heads), 2);
  const int groups = a.c.block / 4 * (a.c.d / 8);      // at most so many in a page
  if (a.longest == 1) hipLaunchKernelGGL((append_kernel<Tag, kFewThreads, 1>), grid, dim3(kFewThreads), 0, st, a);
  else if (groups <= kThreads) hipLaunchKernelGGL((append_kernel<Tag, kThreads, 1>), grid, dim3(kThreads), 0, st, a);
  else if (groups <= 2 * kThreads) hipLaunchKernelGGL((append_kernel<Tag, kThreads, 2>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((append_kernel<Tag, kThreads, 4>), grid, dim3(kThreads), 0, st, a);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
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
  hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == CAFEQ_F32 ? launch_append<F32Tag>(a, st) : launch_append<BF16Tag>(a, st);
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
