// Attention of many new tokens a sequence over the 8-bit cache: prompts, and chunks of them.
#include "attend.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kJoin = 256;

// What of a lane's row is rarely looked at, in LDS, [what][thread]: the registers serve the tiles.  Keys in its reach; its reference where scores are large;
// the maximum and the sum of keys on pages of zeros
enum RowPart { kFirstKey, kEndKey, kBase, kZeroMax, kZeroSum, kRowParts };

__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

// A workgroup: 32 rows a wave, over a part of the keys, in tiles of KT.  A tile's codes are read once, become float16 on their way to LDS
// and are what all waves multiply: v_mfma 32x32x16, S^T = K Q^T with the rows of q in registers, then out^T = V^T P^T.  Lane l holds row l % 32,
// and of 32 keys those with key / 4 % 2 = l / 32: results i of a product are keys 8 (i / 4) + 4 (l / 32) + i % 4, weights 8 u .. 8 u + 7 what it gives to step u of
// the second product.  LDS: K as [16 channels][half][key], V as [16 keys][half][channel] of eight float16 each, a place of 16 bytes
// behind every run so that lanes that write side by side hit different banks.  Two buffers: the next tile's codes are on their way while this one is multiplied.
// Bound by what a wave does one after another: products, exponentials (at a quarter of the rate, two and a reciprocal with a soft cap), reads of LDS: a prompt of 8192,
// 8 heads of 256, 16 query heads 667 us, 824 TFLOP/s, with a soft cap 758 (replayed on one state; 803 on three in turn); 16 heads of 128, 32 query heads 643, 855 TFLOP/s; a product of
// 8192^3 reaches 1360.  Counted: of heads of 256 with a cap the matrix pipe is busy 32 % of the time, vector instructions issue in 40 % (exponentials and reciprocals take four times as
// long), LDS is active in 22 %; of heads of 128 39, 63 and 40 %.  Nothing is saturated: waves leave a barrier in step, and what they do adds up.  Raised priority around
// the matrix instructions, or around the rest, made it 5 to 18 % slower; operands read four steps ahead nothing; 64 rows a wave (half the LDS reads) spilled.
// ONE: a tile's keys are of one page.
template <class Tag, int DB, bool EXACT, bool ONE>
__global__ __launch_bounds__(64 * many_waves(Tag::dtype, DB), many_resident(Tag::dtype, DB)) void attend_many_kernel(const AttendPlan p) {
  using elem = typename Tag::elem;
  constexpr bool kF32 = Tag::dtype == CAFEQ_F32;
  constexpr int kWaves = many_waves(Tag::dtype, DB), kThreads = 64 * kWaves, kParts = kF32 ? 2 : 1, KT = many_keys(Tag::dtype, DB), NT = KT / 32;
  constexpr int KS = 4 * DB, MT = 2 * DB, U = KT / 16, kTile = 32 * kWaves, E = (KT * KS + kThreads - 1) / kThreads;
  constexpr int kRunK = KT + 1, kRunV = 64 * DB + 1, kBufK = 2 * KS * kRunK, kBuf = kBufK + 2 * U * kRunV;
  extern __shared__ __align__(16) half8_t buf[];
  const cafeq_cache& c = p.c;
  const cafeq_attention& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x % c.heads, split = blockIdx.y, shift_b = p.shift, B = c.block, d = EXACT ? 64 * DB : c.d, chunks = d / 16;
  // later rows of a sequence reach more keys: first
  const int64_t w = (gridDim.x - 1 - blockIdx.x) / c.heads;
  const int i = sequence_of(p.units, a.starts, c.sequences, int(a.n), w);
  if (i < 0) return;
  // (starts out of order may put it anywhere: rows are below 2^31)
  const int first = int(min(w - p.units.base(min(max(a.starts[i], 0), int(a.n)), i), int64_t(INT32_MAX / kTile))) * kTile;
  const Reach r = reach_of(c, a, i, p.rep, first, kTile);
  if (first >= r.rows || r.rows <= p.few_rows) return;
  const int c0 = r.lo / KT, c1 = max(c0, (r.hi + KT - 1) / KT), used = max(1, (c1 - c0 + p.span - 1) / p.span);
  if (split >= used) return;
  const int begin = c0 + split * p.span, end = min(c1, begin + p.span);

  // rows of the wave
  const int wfirst = first + wave * 32, wlast = min(wfirst + 32, r.rows) - 1;
  const int wlo = key_begin(a, r.pos0 + wfirst / p.rep), whi = wlast < wfirst ? 0 : key_end(a, r.len, r.pos0 + wlast / p.rep);
  const int all_lo = key_begin(a, r.pos0 + max(wlast, 0) / p.rep), all_hi = key_end(a, r.len, r.pos0 + wfirst / p.rep);
  half8_t q[kParts][KS];
  const int mine = wfirst + l32, token = mine / p.rep, pos = r.pos0 + token;
  const bool live = mine < r.rows;
  const int klo = live ? key_begin(a, pos) : 0, khi = live ? key_end(a, r.len, pos) : 0;
  const elem* qrow = static_cast<const elem*>(a.q) + int64_t(r.row0 + (live ? token : 0)) * a.ldq + int64_t(head * p.rep + (live ? mine - token * p.rep : 0)) * a.hsq;
  float v[KS][8];
  uint32_t bits = 0;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const bool in = live && (EXACT || 16 * s < d);
    const elem* y = qrow + (EXACT || 16 * s < d ? 16 * s + 8 * h : 0);
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 f = load4(y + e);
      v[s][e] = in ? f.x : 0.f; v[s][e + 1] = in ? f.y : 0.f; v[s][e + 2] = in ? f.z : 0.f; v[s][e + 3] = in ? f.w : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) bits = max(bits, __float_as_uint(v[s][e]) & 0x7FFFFFFFu);
  }
  bits = max(bits, uint32_t(__shfl_xor(int(bits), 32)));
  const QueryScale qs = query_scale(bits, a);
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float f0 = v[s][e] * qs.up, f1 = v[s][e + 1] * qs.up;
      const half2_t x2 = to_half(f0, f1);
      q[0][s][e] = x2[0];
      q[0][s][e + 1] = x2[1];
      if constexpr (kF32) {
        const half2_t y2 = to_half(f0 - float(x2[0]), f1 - float(x2[1]));
        q[1][s][e] = y2[0];
        q[1][s][e + 1] = y2[1];
      }
    }

  // what this thread brings of every tile: 16 channels of a key, 16 keys of a channel
  const int32_t* table = c.table + int64_t(i) * c.width;
  int kkey[E], kat[E], klds[E], vrun[E], vat[E], vlds[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int n = tid + e * kThreads, key = min(n / chunks, KT - 1), s = n % chunks;
    kkey[e] = key;
    kat[e] = key * d + 16 * s;
    klds[e] = n < KT * chunks ? 2 * s * kRunK + key : -1;
    const int u = n % U, ch = min(n / U, d - 1);
    vrun[e] = 16 * u;
    vat[e] = ch * B;
    vlds[e] = n < U * d ? kBufK + 2 * u * kRunV + ch : -1;
  }
  auto page_at = [&](int key) {
    const int entry = table[min(key >> shift_b, c.width - 1)];
    return key < r.len && entry >= 0 && entry < c.pages ? entry : -1;
  };
  int kpage[E], vpage[E], spage;     // pages of the tile that is requested next; lanes 0 .. U - 1 hold those of its runs of 16 keys
  auto pages_of = [&](int tile) {
    if constexpr (ONE) {
      spage = page_at(tile * KT);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        kpage[e] = page_at(tile * KT + kkey[e]);
        vpage[e] = page_at(tile * KT + vrun[e]);
      }
      spage = page_at(tile * KT + 16 * (lane & (U - 1)));
    }
  };
  uint4 kc[E], vc[E];
  float ks, vs;
  bool hole;
  auto request = [&](int tile) {
    const int in_page = B - 1;
    if constexpr (ONE) {
      // one page: its place is the wave's, a thread's part of it stays
      const int page = __builtin_amdgcn_readfirstlane(spage), key = (tile * KT) & in_page;
      const int64_t at = int64_t(max(page, 0)) * c.heads + head;
      const int8_t *k = c.k + (at * B + key) * d, *v = c.v + at * B * d + key;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        kc[e] = *reinterpret_cast<const uint4*>(k + uint32_t(kat[e]));
        vc[e] = *reinterpret_cast<const uint4*>(v + uint32_t(vat[e] + vrun[e]));
      }
      ks = c.kscale[at];
      vs = c.vscale[at];
      hole = page < 0;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        // key * d + channel within the page: the tile's first key may lie inside a page, and a page inside the tile
        const int8_t* k = c.k + (int64_t(max(kpage[e], 0)) * c.heads + head) * B * d;
        const int key = (tile * KT + kkey[e]) & in_page;
        kc[e] = *reinterpret_cast<const uint4*>(k + key * d + (kat[e] - kkey[e] * d));
        const int8_t* v = c.v + (int64_t(max(vpage[e], 0)) * c.heads + head) * B * d;
        vc[e] = *reinterpret_cast<const uint4*>(v + vat[e] + ((tile * KT + vrun[e]) & in_page));
      }
      const int64_t s = int64_t(max(spage, 0)) * c.heads + head;
      ks = c.kscale[s];
      vs = c.vscale[s];
      hole = spage < 0;
    }
  };
  auto put = [&](half8_t* to) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (klds[e] >= 0) {
        to[klds[e]] = half_codes(kc[e].x, kc[e].y);
        to[klds[e] + kRunK] = half_codes(kc[e].z, kc[e].w);
      }
      if (vlds[e] >= 0) {
        to[vlds[e]] = half_codes(vc[e].x, vc[e].z);
        to[vlds[e] + kRunV] = half_codes(vc[e].y, vc[e].w);
      }
    }
  };

  f32x16_t o[MT];
  float M = kNoKey, l = 0.f;
  float* row_lds = reinterpret_cast<float*>(buf + 2 * kBuf) + tid;
  auto row = [&](int what) -> float& { return row_lds[what * kThreads]; };
  // scales of k (their bits) from which on scores of the wave's rows may be large, or take the cap of large ones; 0 once a row has a reference
  float most_unit = fmaxf(0.f, qs.unit);
#pragma unroll
  for (int k = 1; k < 32; k <<= 1) most_unit = fmaxf(most_unit, __shfl_xor(most_unit, k));
  const uint32_t near_scale = __builtin_amdgcn_readfirstlane(p.cap == kCapWide ? 1u : p.cap == kCapNear && p.cap_out <= kFar ? 0xFFFFFFFFu :
                                                             max(1u, __float_as_uint(near_factor(DB) / most_unit)));
  uint32_t far_scale = near_scale;
  row(kFirstKey) = __int_as_float(klo);
  row(kEndKey) = __int_as_float(khi);
  row(kZeroMax) = kNoKey;
  row(kZeroSum) = 0.f;
#pragma unroll
  for (int m = 0; m < MT; ++m) o[m] = f32x16_t{};

  if (begin < end) {
    pages_of(begin);
    request(begin);
    pages_of(begin + 1);
    put(buf);
  }
  __syncthreads();
  for (int tile = begin; tile < end; ++tile) {
    const half8_t* now_buf = buf + ((tile - begin) & 1) * kBuf;
    const float tks = ks, tvs = vs;
    const bool thole = hole;
    if (tile + 1 < end) {
      request(tile + 1);
      pages_of(tile + 2);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int key0 = tile * KT + 32 * n;
      if (key0 >= whi || key0 + 32 <= wlo) continue;
      f32x16_t x = f32x16_t{};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if (!EXACT && 16 * s >= d) continue;
        const half8_t k = now_buf[(2 * s + h) * kRunK + 32 * n + l32];
#pragma unroll
        for (int e = kParts - 1; e >= 0; --e) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[e][s], x, 0, 0, 0);
      }
      // runs of 16 keys, results 0 .. 7 and 8 .. 15, which may be of two pages
      constexpr int kRuns = ONE ? 1 : 2, kRun = 16 / kRuns;
      ValueScale sc[kRuns];
      float ksc[kRuns];
      bool gone[kRuns], far = false, odd = key0 < all_lo || key0 + 32 > all_hi;
#pragma unroll
      for (int k = 0; k < kRuns; ++k) {
        const int at = ONE ? 0 : 2 * n + k;
        ksc[k] = lane_value(tks, at);
        sc[k] = value_scale(lane_value(tvs, at));
        gone[k] = __builtin_amdgcn_readlane(int(thole), at);
        far |= __float_as_uint(ksc[k]) >= far_scale;
        odd |= gone[k] || sc[k].zero || !(ksc[k] >= 0.f) || far;
        if constexpr (!kF32) {
          // the mantissa goes into the exponent too: one rounding of the argument for the page, for a multiplication a weight
          sc[k].exp += __builtin_amdgcn_logf(sc[k].mant);
          sc[k].inv *= __builtin_amdgcn_rcpf(sc[k].mant);
        }
      }
      half8_t wt[kParts][2];
      float f[kRuns];
#pragma unroll
      for (int k = 0; k < kRuns; ++k) f[k] = qs.unit * ksc[k];
      if (p.cap == kCapNear) {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = capped<kF32>(x[e] * (f[e / kRun] * p.cap_in), p.cap_out);
#pragma unroll
        for (int k = 0; k < kRuns; ++k) f[k] = 1.f;
      }
      float top = kNoKey;
      int from = 0, to = 0;
      if (__builtin_expect(odd, 0)) {
        from = __float_as_int(row(kFirstKey)) - key0 - 4 * h;
        to = __float_as_int(row(kEndKey)) - key0 - 4 * h;
      }
      auto in = [&](int e) { return bool(int(8 * (e >> 2) + (e & 3) >= from) & int(8 * (e >> 2) + (e & 3) < to) & int(!gone[e / kRun])); };
      if (__builtin_expect(!odd, 1)) {
#pragma unroll
        for (int k = 0; k < kRuns; ++k) {
          float y = x[kRun * k];
#pragma unroll
          for (int e = 1; e < kRun; ++e) y = fmaxf(y, x[kRun * k + e]);
          top = fmaxf(top, fmaf(y, f[k], sc[k].exp));
        }
      } else {
        if (__builtin_expect(far, 0)) {
          if (p.cap == kCapWide) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = capped_wide(x[e] * (f[e / kRun] * p.cap_in), p.cap_out);
#pragma unroll
            for (int k = 0; k < kRuns; ++k) f[k] = 1.f;
          }
          float high = kNoKey;
#pragma unroll
          for (int e = 0; e < 16; ++e) high = int(in(e)) & int(!sc[e / kRun].zero) ? fmaxf(high, x[e] * f[e / kRun]) : high;
          const float old = far_scale == 0u ? row(kBase) : 0.f, base = next_base(other_half(high), old, M == kNoKey);
          M = M == kNoKey ? M : M + (old - base);
          far_scale = __ballot(base != 0.f) ? 0u : near_scale;
          if (far_scale == 0u) row(kBase) = base;
          if (base != 0.f) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = x[e] * f[e / kRun] - (sc[e / kRun].zero ? 0.f : base);
#pragma unroll
            for (int k = 0; k < kRuns; ++k) f[k] = 1.f;
          }
        }
#pragma unroll
        for (int k = 0; k < kRuns; ++k) {
          float y = kNoKey;
#pragma unroll
          for (int e = kRun * k; e < kRun * k + kRun; ++e) y = in(e) ? fmaxf(y, x[e]) : y;
          if (sc[k].zero) {
            // keys of a page of zeros count in the sum of weights only, on a maximum of their own
            float mz = row(kZeroMax), lz = row(kZeroSum);
            const float most = fmaxf(mz, other_half(y == kNoKey ? y : y * f[k]));
            lz *= __builtin_amdgcn_exp2f(mz - most);
            mz = most;
#pragma unroll
            for (int e = kRun * k; e < kRun * k + kRun; ++e) lz += in(e) ? __builtin_amdgcn_exp2f(x[e] * f[k] - most) : 0.f;
            row(kZeroMax) = mz;
            row(kZeroSum) = lz;
          } else {
            top = y == kNoKey ? top : fmaxf(top, fmaf(y, f[k], sc[k].exp));
          }
        }
      }
      const float most = fmaxf(M, ceilf(other_half(top)) - kTop);
      if (__ballot(most != M)) {
        const float back = __builtin_amdgcn_exp2f(M - most);
        l *= back;
#pragma unroll
        for (int m = 0; m < MT; ++m) o[m] *= back;
        M = most;
      }
      float P[16];
#pragma unroll
      for (int k = 0; k < kRuns; ++k) {
        const float shift = sc[k].exp - M;
        float sum = 0.f;
#pragma unroll
        for (int e = kRun * k; e < kRun * k + kRun; ++e) P[e] = __builtin_amdgcn_exp2f(fmaf(x[e], f[k], shift));
        if (__builtin_expect(odd, 0)) {      // a scale that is no number must not reach keys that do not count
#pragma unroll
          for (int e = kRun * k; e < kRun * k + kRun; ++e) P[e] = int(in(e)) & int(!sc[k].zero) ? P[e] : 0.f;
        }
#pragma unroll
        for (int e = kRun * k; e < kRun * k + kRun; ++e) sum += P[e];
        if constexpr (kF32) {
#pragma unroll
          for (int e = kRun * k; e < kRun * k + kRun; ++e) P[e] *= sc[k].mant;
          if (__builtin_expect(odd, 0)) {
#pragma unroll
            for (int e = kRun * k; e < kRun * k + kRun; ++e) P[e] = int(in(e)) & int(!sc[k].zero) ? P[e] : 0.f;
          }
        }
        l = sum == 0.f ? l : fmaf(sum, sc[k].inv, l);      // (nothing times a scale that is no number is nothing)
      }
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const half2_t y = to_half(P[e], P[e + 1]);
        wt[0][e >> 3][e & 7] = y[0];
        wt[0][e >> 3][(e & 7) + 1] = y[1];
        if constexpr (kF32) {
          const half2_t rest = to_half(P[e] - float(y[0]), P[e + 1] - float(y[1]));
          wt[1][e >> 3][e & 7] = rest[0];
          wt[1][e >> 3][(e & 7) + 1] = rest[1];
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if (!EXACT && 32 * m >= d) continue;
          const half8_t v = now_buf[kBufK + (2 * (2 * n + u) + h) * kRunV + 32 * m + l32];
#pragma unroll
          for (int e = kParts - 1; e >= 0; --e) o[m] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, wt[e][u], o[m], 0, 0, 0);
        }
    }
    if (tile + 1 < end) put(buf + ((tile + 1 - begin) & 1) * kBuf);
    __syncthreads();
  }

  const int64_t part = ((w * c.heads + head) * p.splits + split) * kTile;
  const int place = wave * 32 + l32, R = first + place;
  float sum = l + __shfl_xor(l, 32), lz = row(kZeroSum), sumz = lz + __shfl_xor(lz, 32), mz = row(kZeroMax);
  const Finish fin = finish_of(M, far_scale == 0u ? row(kBase) : 0.f);
  const float both = fmaxf(fin.all, mz), near = __builtin_amdgcn_exp2f(fin.all - both), own = fin.unit * near;
  const float total = sum * (fin.sum_unit * near) + sumz * __builtin_amdgcn_exp2f(mz - both);
  if (R >= r.rows) return;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int ch = 32 * m + 2 * e + 4 * h;
      if (!EXACT && ch >= d) continue;
      const f32x4_t v = f32x4_t{o[m][e], o[m][e + 1], o[m][e + 2], o[m][e + 3]} * own;
      if (used > 1) *reinterpret_cast<f32x4_t*>(p.parts + (part + place) * d + ch) = v;
      else store_row<Tag>(p, r, R, head, ch, v, both, total);
    }
  if (used > 1 && h == 0) *reinterpret_cast<float2*>(p.sums + 2 * (part + place)) = make_float2(both, total);
}

// The parts of a tile's rows joined in their order, four channels a thread.
template <class Tag, int DB>
__global__ __launch_bounds__(kJoin) void attend_many_join_kernel(const AttendPlan p) {
  constexpr int kTile = 32 * many_waves(Tag::dtype, DB), KT = many_keys(Tag::dtype, DB);
  const cafeq_cache& c = p.c;
  const int head = blockIdx.x % c.heads, d = c.d, per = d / 4;
  const int64_t w = blockIdx.x / c.heads;
  const int i = sequence_of(p.units, p.a.starts, c.sequences, int(p.a.n), w);
  if (i < 0) return;
  const int first = int(min(w - p.units.base(min(max(p.a.starts[i], 0), int(p.a.n)), i), int64_t(INT32_MAX / kTile))) * kTile;
  const Reach r = reach_of(c, p.a, i, p.rep, first, kTile);
  if (first >= r.rows || r.rows <= p.few_rows) return;
  const int c0 = r.lo / KT, c1 = max(c0, (r.hi + KT - 1) / KT), used = (c1 - c0 + p.span - 1) / p.span;
  const int e = blockIdx.y * kJoin + threadIdx.x, row = e / per, ch = e % per * 4;
  if (used <= 1 || row >= kTile || first + row >= r.rows) return;
  const int64_t part = (w * c.heads + head) * p.splits * kTile + row;
  float big = kNoKey, total = 0.f;
  for (int s = 0; s < used; ++s) big = fmaxf(big, p.sums[2 * (part + int64_t(s) * kTile)]);
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < used; ++s) {
    const int64_t at = part + int64_t(s) * kTile;
    const float2 m = *reinterpret_cast<const float2*>(p.sums + 2 * at);
    const float f = __builtin_amdgcn_exp2f(m.x - big);
    total += m.y * f;
    v += *reinterpret_cast<const f32x4_t*>(p.parts + at * d + ch) * f;
  }
  store_row<Tag>(p, r, first + row, head, ch, v, big, total);
}

template <class Tag, int DB, bool EXACT, bool ONE>
int launch_one(const AttendPlan& p, hipStream_t st) {
  constexpr int KT = many_keys(Tag::dtype, DB), kWaves = many_waves(Tag::dtype, DB), kTile = 32 * kWaves;
  constexpr size_t lds = 2 * 16 * (2 * 4 * DB * (KT + 1) + 2 * (KT / 16) * (64 * DB + 1)) + sizeof(float) * kRowParts * 64 * kWaves;
  const auto kern = attend_many_kernel<Tag, DB, EXACT, ONE>;
  if (lds > 65536) {
    static const bool ok = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds)) == hipSuccess;
    if (!ok) return CAFEQ_ERR_LAUNCH;
  }
  // the heads innermost: workgroups go round the eight XCDs in turn, so that a head's tiles stay behind one L2
  const unsigned units = unsigned(p.units.count(p.a.n, p.c.sequences) * p.c.heads);
  hipLaunchKernelGGL(kern, dim3(units, unsigned(p.splits)), dim3(64 * kWaves), lds, st, p);
  CAFEQ_CHECK_LAUNCH();
  if (p.splits > 1) {
    const unsigned y = unsigned((kTile * (p.c.d / 4) + kJoin - 1) / kJoin);
    hipLaunchKernelGGL((attend_many_join_kernel<Tag, DB>), dim3(units, y), dim3(kJoin), 0, st, p);
    CAFEQ_CHECK_LAUNCH();
  }
  return CAFEQ_OK;
}

template <class Tag, int DB, bool EXACT>
int launch(const AttendPlan& p, hipStream_t st) {
  return p.c.block >= many_keys(Tag::dtype, DB) ? launch_one<Tag, DB, EXACT, true>(p, st) : launch_one<Tag, DB, EXACT, false>(p, st);
}

template <class Tag>
int launch_type(const AttendPlan& p, hipStream_t st) {
  switch (p.c.d) {
    case 64: return launch<Tag, 1, true>(p, st);
    case 128: return launch<Tag, 2, true>(p, st);
    case 256: return launch<Tag, 4, true>(p, st);
  }
  switch ((p.c.d + 63) / 64) {
    case 1: return launch<Tag, 1, false>(p, st);
    case 2: return launch<Tag, 2, false>(p, st);
    case 3: return launch<Tag, 3, false>(p, st);
    default: return launch<Tag, 4, false>(p, st);
  }
}

}  // namespace

int launch_attend_many(const AttendPlan& p, hipStream_t st) {
  return p.a.dtype == CAFEQ_F32 ? launch_type<F32Tag>(p, st) : launch_type<BF16Tag>(p, st);
}

}  // namespace cafeq
