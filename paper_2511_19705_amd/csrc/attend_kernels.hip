// Attention of new tokens over the cache in 8 bits.
#include "cache.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kThreads = 256;

struct AttendArgs {
  cafeq_cache c;
  cafeq_attention a;
};

// A wave a row and query head, one key at a time: lane l holds channels 4 l .. 4 l + 3.
template <class Tag>
__global__ __launch_bounds__(kThreads) void attend_kernel(const AttendArgs p) {
  using elem = typename Tag::elem;
  const cafeq_cache& c = p.c;
  const cafeq_attention& a = p.a;
  const int lane = threadIdx.x & 63, n = int(a.n), B = c.block, d = c.d;
  const int64_t unit = int64_t(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  const int row = int(unit / a.heads_q), h = int(unit % a.heads_q);
  if (row >= n) return;
  const int i = sequence_of(Units{1, 1, 0}, a.starts, c.sequences, n, row);
  if (i < 0) return;
  const RowRange r = rows_of(a.starts, i, n);
  if (row >= r.hi || row - r.lo >= a.longest) return;
  const int len = tokens_of(c, i), pos = len - (r.hi - row), kv = h / (a.heads_q / c.heads);
  const int hi = a.causal ? min(len, pos + 1) : len, lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  const bool in = 4 * lane < d;
  const elem* q = static_cast<const elem*>(a.q) + row * a.ldq + h * a.hsq;
  float4 x = in ? load4(q + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
  if (__ballot(!isfinite(x.x) || !isfinite(x.y) || !isfinite(x.z) || !isfinite(x.w))) x.x = NAN;
  // sums over 64 keys, and sums of those: thousands of keys one after another would cost float32's last bits
  float M = -FLT_MAX, L = 0.f, O[4] = {0.f, 0.f, 0.f, 0.f}, m = -FLT_MAX, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  auto join = [&]() {
    const float top = fmaxf(M, m), f = expf(M - top), g = expf(m - top);
    M = top;
    L = L * f + l * g;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      O[j] = O[j] * f + o[j] * g;
      o[j] = 0.f;
    }
    m = -FLT_MAX;
    l = 0.f;
  };
  for (int t = lo; t < hi; ++t) {
    if ((t & 63) == 0) join();
    const int page = page_of(c, i, t / B);
    if (page < 0) continue;
    const int64_t at = int64_t(page) * c.heads + kv;
    const int slot = t % B;
    float s = 0.f;
    if (in) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(c.k + (at * B + slot) * d + 4 * lane);
      s = x.x * float(int8_t(w)) + x.y * float(int8_t(w >> 8)) + x.z * float(int8_t(w >> 16)) + x.w * float(int8_t(w >> 24));
    }
    s = wave_sum(s) * (c.kscale[at] * a.scale);
    if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
    const float top = fmaxf(m, s), f = expf(m - top), e = expf(s - top);
    m = top;
    l = l * f + e;
    const float ev = e * c.vscale[at];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] * f + (in ? ev * float(c.v[(at * d + 4 * lane + j) * B + slot]) : 0.f);
  }
  join();
  const float inv = L == 0.f ? 0.f : 1.f / L;
  elem* y = static_cast<elem*>(a.out) + row * a.ldo + h * a.hso + 4 * lane;
  if (in) {
    if constexpr (Tag::dtype == CAFEQ_F32) *reinterpret_cast<float4*>(y) = make_float4(O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv);
    else *reinterpret_cast<uint2*>(y) = make_uint2(bf16_bits(O[0] * inv, O[1] * inv), bf16_bits(O[2] * inv, O[3] * inv));
  }
  if (a.lse && lane == 0) a.lse[int64_t(row) * a.heads_q + h] = L == 0.f ? -INFINITY : M + logf(L);
}

int check_attention(const cafeq_cache* c, const cafeq_attention* a) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!a || !a->q || !a->out || !a->starts || (a->dtype != CAFEQ_F32 && a->dtype != CAFEQ_BF16)) return CAFEQ_ERR_INVALID_ARG;
  if (a->n < 0 || a->longest < 0 || a->heads_q < 1 || a->heads_q % c->heads || a->window < 0 || !(a->softcap >= 0.f) || a->ldq < 0 || a->hsq < 0)
    return CAFEQ_ERR_BAD_SHAPE;
  if (a->n > (int64_t(1) << 24) || a->heads_q > kMaxHeads || a->n * a->heads_q > INT32_MAX) return CAFEQ_ERR_UNSUPPORTED;
  const int size = a->dtype == CAFEQ_F32 ? 4 : 2;
  if (!aligned_to(a->q, 16) || !aligned_to(a->out, 16) || (a->ldq | a->hsq | a->ldo | a->hso) % (16 / size) || !aligned_to(a->starts, 4) ||
      !aligned_to(a->lse, 4))
    return CAFEQ_ERR_BAD_ALIGN;
  const HeadRows q{a->q, a->n, a->ldq, a->heads_q, a->hsq, c->d, size}, o{a->out, a->n, a->ldo, a->heads_q, a->hso, c->d, size};
  if (a->n > 0 && !o.plain()) return CAFEQ_ERR_BAD_SHAPE;
  if (may_share(q, o)) return CAFEQ_ERR_INVALID_ARG;
  return CAFEQ_OK;
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_cache_attend_workspace_bytes(const cafeq_cache* cache, const cafeq_attention* a) {
  if (check_attention(cache, a)) return 0;
  return 0;
}

int cafeq_cache_attend(const cafeq_cache* cache, const cafeq_attention* a, void* ws, void* stream) {
  const int rc = check_attention(cache, a);
  if (rc) return rc;
  if (!aligned_to(ws, 16)) return CAFEQ_ERR_BAD_ALIGN;
  if (a->n == 0 || a->longest == 0 || cache->sequences == 0) return CAFEQ_OK;
  const AttendArgs p{*cache, *a};
  const dim3 grid(unsigned((a->n * a->heads_q + 3) / 4));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a->dtype == CAFEQ_F32) hipLaunchKernelGGL((attend_kernel<F32Tag>), grid, dim3(kThreads), 0, st, p);
  else hipLaunchKernelGGL((attend_kernel<BF16Tag>), grid, dim3(kThreads), 0, st, p);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

}  // extern "C"
