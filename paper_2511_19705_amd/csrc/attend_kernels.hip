// Attention of new tokens over the cache in 8 bits.
#include "attend.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

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

// How the rows and keys are cut.  Sums and parts lie behind each other in the workspace.
AttendPlan plan(const cafeq_cache& c, const cafeq_attention& a) {
  AttendPlan p{c, a, a.heads_q / c.heads, __builtin_ctz(unsigned(c.block))};
  p.a.longest = std::min(a.longest, a.n);
  const int64_t rows = p.a.longest * p.rep, room = int64_t(c.width) * c.block;
  p.tiles = int((rows + 15) / 16);
  p.keep = int(std::min<int64_t>(16, rows));
  // keys that a tile may reach
  const int64_t keys = a.window > 0 && a.causal ? std::min(room, a.window + 16 + int64_t(128)) : room;
  const int64_t groups = int64_t(c.sequences) * p.tiles * c.heads;
  // Two workgroups a compute unit at once, but none with less than 128 keys (a step a wave) or more than 2048 (lengths differ); half as long where
  // that leaves few to choose from.  us with 128 / 256 / 512 keys: 512 of 4 heads of 256 11.3 / 13.6 / 14.8, 4096 12.0 / 13.7 / 18.2; 32768 of 8 heads with
  // 256 / 512 / 1024 keys 36 / 31.5 / 33; 48 x 8192 of 8 heads with 1024 / 2048 / 4096 318 / 302 / 323; 32 x 4096 of 4 heads, two row tiles, with
  // 1024 / 2048 60 / 76.
  int64_t part = std::min<int64_t>(2048, std::max<int64_t>(128, keys * groups / 512));
  while (part > 512 && keys * groups / part < 1024) part /= 2;
  p.span = int((part + 31) / 32);
  p.span = std::max<int>(p.span, int((keys + int64_t(32) * 65535 - 1) / (int64_t(32) * 65535)));      // a grid's second dimension
  p.splits = int((keys + 32 * int64_t(p.span) - 1) / (32 * int64_t(p.span)));
  if (p.c.heads % 8 && p.splits % 2 == 0) ++p.splits;      // so that sequences begin on different XCDs
  return p;
}
size_t sums_bytes(const AttendPlan& p) {
  return align_up(size_t(p.c.sequences) * p.tiles * p.c.heads * p.splits * p.keep * 2 * sizeof(float), 256);
}
size_t plan_bytes(const AttendPlan& p) { return p.splits > 1 ? sums_bytes(p) + sums_bytes(p) / 2 * size_t(p.c.d) : 0; }

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_cache_attend_workspace_bytes(const cafeq_cache* cache, const cafeq_attention* a) {
  if (check_attention(cache, a) || a->n == 0 || a->longest == 0 || cache->sequences == 0) return 0;
  return plan_bytes(plan(*cache, *a));
}

int cafeq_cache_attend(const cafeq_cache* cache, const cafeq_attention* a, void* ws, void* stream) {
  const int rc = check_attention(cache, a);
  if (rc) return rc;
  if (!aligned_to(ws, 16)) return CAFEQ_ERR_BAD_ALIGN;
  if (a->n == 0 || a->longest == 0 || cache->sequences == 0) return CAFEQ_OK;
  AttendPlan p = plan(*cache, *a);
  if (plan_bytes(p)) {
    if (!ws) return CAFEQ_ERR_WORKSPACE;
    p.sums = static_cast<float*>(ws);
    p.parts = p.sums + sums_bytes(p) / sizeof(float);
  }
  return launch_attend_few(p, static_cast<hipStream_t>(stream));
}

}  // extern "C"
