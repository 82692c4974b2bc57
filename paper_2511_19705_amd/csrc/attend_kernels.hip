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

// Rows of a sequence and key head up to which attend_few is the faster, though it reads the keys once for every 16: 8 x 3000 keys of 16 heads of 128, 64 rows,
// 79 us in four tiles of 16 and 60 by attend_many; of 8 heads of 256 64 and 81; 60000 keys of 8 heads of 256, 32 rows 75 and 150, 128 rows 239 and 172.
int64_t few_rows(const cafeq_cache& c) { return c.d > 128 ? 64 : 32; }

size_t sums_bytes(const AttendPlan& p, int64_t tiles) {
  return p.splits > 1 ? align_up(size_t(tiles) * p.c.heads * p.splits * p.keep * 2 * sizeof(float), 256) : 0;
}
size_t parts_bytes(const AttendPlan& p, int64_t tiles) { return sums_bytes(p, tiles) / 2 * size_t(p.c.d); }

// How rows and keys are cut.  Sequences with up to few_rows rows a key head go to attend_few, the others to attend_many; one launch where the bound on
// their tokens, or a single sequence, leaves no doubt.
struct AttendPlans {
  bool few, many;
  AttendPlan f, m;
  int64_t few_tiles, many_tiles;
  size_t few_sums, few_parts, many_sums, many_parts;
  size_t bytes() const { return few_sums + few_parts + many_sums + many_parts; }
  // a launch's first dimension holds less than 2^32 threads
  bool fits() const { return !many || many_tiles * m.c.heads * 64 * many_waves(m.a.dtype, (m.c.d + 63) / 64) <= int64_t(UINT32_MAX); }
};

AttendPlan plan_of(const cafeq_cache& c, const cafeq_attention& a) {
  AttendPlan p{c, a, a.heads_q / c.heads, __builtin_ctz(unsigned(c.block))};
  if (a.softcap > 0.f) {
    // a cap below 2^-30 leaves every score within 2^-30 of 0, however steep the way there
    const float in = std::min(1.f / a.softcap, 0x1p30f);
    p.cap = a.dtype != CAFEQ_F32 && a.softcap > kWideCap ? kCapWide : kCapNear;
    p.cap_in = a.dtype == CAFEQ_F32 ? in : 2.f * kLog2e * in;
    p.cap_out = a.softcap * kLog2e;
  }
  return p;
}

AttendPlan plan_few(const cafeq_cache& c, const cafeq_attention& a, int64_t rows, int64_t room) {
  AttendPlan p = plan_of(c, a);
  p.few_rows = int(std::min<int64_t>(rows, INT32_MAX));
  p.tiles = int((rows + 15) / 16);
  p.keep = int(std::min<int64_t>(16, rows));
  // keys that a tile may reach
  const int64_t keys = a.window > 0 && a.causal ? std::min(room, a.window + int64_t(16 + 128)) : room;
  const int64_t groups = int64_t(c.sequences) * p.tiles * c.heads;
  // Two workgroups a compute unit at once, but none with less than 128 keys (a step a wave) or more than 2048 (lengths differ); half as long where
  // that leaves few to choose from.  us with 128 / 256 / 512 keys: 512 of 4 heads of 256 11.3 / 13.6 / 14.8, 4096 12.0 / 13.7 / 18.2; 32768 of 8 heads with
  // 256 / 512 / 1024 keys 36 / 31.5 / 33; 48 x 8192 of 8 heads with 1024 / 2048 / 4096 318 / 302 / 323; 32 x 4096 of 4 heads, two row tiles, with
  // 1024 / 2048 60 / 76.
  int64_t part = std::min<int64_t>(2048, std::max<int64_t>(128, keys * groups / 512));
  while (part > 512 && keys * groups / part < 1024) part /= 2;
  // room that sequences do not use is cut too, into workgroups that end at once: not too many of them
  while (part < keys && keys * groups / part > 16384) part *= 2;
  p.span = int((part + 31) / 32);
  p.span = std::max<int>(p.span, int((keys + int64_t(32) * 65535 - 1) / (int64_t(32) * 65535)));      // a grid's second dimension
  p.splits = int((keys + 32 * int64_t(p.span) - 1) / (32 * int64_t(p.span)));
  if (p.c.heads % 8 && p.splits % 2 == 0) ++p.splits;      // so that sequences begin on different XCDs
  return p;
}

AttendPlan plan_many(const cafeq_cache& c, const cafeq_attention& a, int64_t few_rows, int64_t room) {
  AttendPlan p = plan_of(c, a);
  const int db = (c.d + 63) / 64, tile = 32 * many_waves(a.dtype, db), kt = many_keys(a.dtype, db);
  p.few_rows = int(few_rows);
  p.units = Units{p.rep, tile, 1};
  p.keep = tile;
  const int64_t keys = a.window > 0 && a.causal ? std::min(room, a.window + int64_t(tile / p.rep + 2 * kt)) : room;
  const int64_t groups = p.units.count(a.n, c.sequences) * c.heads;
  // workgroups for what the chip holds at once, none with less than 512 keys
  const int64_t slots = int64_t(device_cu_count()) * many_resident(a.dtype, db) * 4 / many_waves(a.dtype, db);
  const int64_t want = std::min((slots + groups - 1) / groups, (keys + 511) / 512);
  p.span = int((keys + want * kt - 1) / (want * kt));
  p.splits = int((keys + int64_t(p.span) * kt - 1) / (int64_t(p.span) * kt));
  return p;
}

AttendPlans plan(const cafeq_cache& c, const cafeq_attention& given) {
  AttendPlans s{};
  cafeq_attention a = given;
  a.longest = std::min(a.longest, a.n);
  if (a.softcap > kNoCap) a.softcap = 0.f;      // bounds nothing: float32 scores below 2^88 keep their bits under it
  if (a.window >= kMaxKeys) a.window = 0;      // reaches all keys: no position is further from the first
  const int64_t rep = a.heads_q / c.heads, rows = a.longest * rep, room = int64_t(c.width) * c.block;
  const int64_t few = few_rows(c);
  s.many = rows > few;
  s.few = !s.many || c.sequences > 1;
  if (s.few) {
    s.f = plan_few(c, a, std::min(rows, few), room);
    s.few_tiles = int64_t(c.sequences) * s.f.tiles;
    s.few_sums = sums_bytes(s.f, s.few_tiles);
    s.few_parts = parts_bytes(s.f, s.few_tiles);
  }
  if (s.many) {
    s.m = plan_many(c, a, s.few ? few : 0, room);
    s.many_tiles = s.m.units.count(a.n, c.sequences);
    s.many_sums = sums_bytes(s.m, s.many_tiles);
    s.many_parts = parts_bytes(s.m, s.many_tiles);
  }
  return s;
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_cache_attend_workspace_bytes(const cafeq_cache* cache, const cafeq_attention* a) {
  if (check_attention(cache, a) || a->n == 0 || a->longest == 0 || cache->sequences == 0) return 0;
  const AttendPlans s = plan(*cache, *a);
  return s.fits() ? s.bytes() : 0;
}

int cafeq_cache_attend(const cafeq_cache* cache, const cafeq_attention* a, void* ws, void* stream) {
  const int rc = check_attention(cache, a);
  if (rc) return rc;
  if (!aligned_to(ws, 16)) return CAFEQ_ERR_BAD_ALIGN;
  if (a->n == 0 || a->longest == 0 || cache->sequences == 0) return CAFEQ_OK;
  AttendPlans s = plan(*cache, *a);
  if (!s.fits()) return CAFEQ_ERR_UNSUPPORTED;
  if (s.bytes() && !ws) return CAFEQ_ERR_WORKSPACE;
  char* at = static_cast<char*>(ws);
  s.f.sums = reinterpret_cast<float*>(at);
  s.f.parts = reinterpret_cast<float*>(at + s.few_sums);
  at += s.few_sums + s.few_parts;
  s.m.sums = reinterpret_cast<float*>(at);
  s.m.parts = reinterpret_cast<float*>(at + s.many_sums);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (s.many) {
    const int rc2 = launch_attend_many(s.m, st);
    if (rc2) return rc2;
  }
  return s.few ? launch_attend_few(s.f, st) : CAFEQ_OK;
}

}  // extern "C"
