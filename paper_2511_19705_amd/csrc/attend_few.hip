// Attention of few new tokens a sequence over the 8-bit cache: memory is the bound, so everything serves the loads.
#include "attend.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kTile = 16, kStep = 32, kWaves = 4, kThreads = 64 * kWaves, kJoin = 256;

// over the four lanes l, l + 16, l + 32, l + 48 that hold a row
__device__ __forceinline__ float across(float v) {
  const uint32_t u = __float_as_uint(v);
  auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const uint32_t w = __float_as_uint(v);
  r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_across(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A workgroup: 16 rows (tokens and query heads that share a key head) over a part of the keys; its waves take steps of 32 keys in turn and
// join in the end.  Lanes l % 16 hold a row, g = l / 16 the keys 16 (g % 2) + 8 (g / 2) .. + 7 of a step: tile t of the first product, v_mfma
// 16x16x32, has the keys of g = r / 4, 4 t + r % 4 of them, in row r, so that a lane's results are the eight keys whose weights it gives to the second
// product.  Codes go from memory to registers, 16 bytes a lane: of k the channels 16 g .. of a key, of v the 16 keys of a run for one channel, of
// which two tiles of 16 channels swap halves between lanes.  The next step's of k are on their way while this one is worked on.
// Bound by memory: 48 sequences of 1600 to 32700 keys, 16 heads of 128, 618 us, 5.4 TB/s (a copy reaches 4.9, reading alone 6.7); one of 131072 109, 4.9 TB/s; 48 of
// 8192, 8 heads of 256, 300, 5.4 TB/s.  Short sequences by what has to follow each other (lengths and pages, codes, two products, the join): 512 keys of 4 heads of
// 256 8.1, and 3.8 for the join.  The rows in LDS and 16 KB of codes a wave at once (8 KB for d of 80, 96 and 112, whose registers are the general form's) keep two waves a
// SIMD, for float32 with d above 192 one.
template <class Tag, int DB, bool EXACT>
__global__ __launch_bounds__(kThreads, Tag::dtype == CAFEQ_F32 && DB == 4 ? 1 : 2) void attend_few_kernel(const AttendPlan p) {
  using elem = typename Tag::elem;
  constexpr bool kF32 = Tag::dtype == CAFEQ_F32;
  constexpr int kParts = kF32 ? 2 : 1, kPairs = 2 * DB;
  constexpr int NS = !EXACT && DB > 1 ? 1 : DB == 1 ? 4 : DB == 2 ? 2 : 1, kKeys = NS * kStep;      // steps a wave takes at once
  extern __shared__ __align__(16) float lds[];
  const cafeq_cache& c = p.c;
  const cafeq_attention& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = blockIdx.z, split = blockIdx.y, tile = p.tiles == 1 ? 0 : blockIdx.x / c.heads, head = blockIdx.x - tile * c.heads;
  const int d = EXACT ? 64 * DB : c.d, B = c.block, shift_b = p.shift, first = tile * kTile, ld = d + 4;
  half8_t* q_lds = reinterpret_cast<half8_t*>(lds);      // [part][64 channels][8 of 16][lane]: the rows as the first product takes them
  float* unit_lds = lds + kParts * DB * 2 * 64 * 4;      // [16]
  float* sum_lds = unit_lds + kTile;                     // [kWaves][16][2]
  float* base_lds = sum_lds + kWaves * kTile * 2;         // [kWaves][16]: references of rows whose scores are large
  float* out_lds = base_lds + kWaves * kTile;             // [kWaves][keep][d + 4]
  const int krun = 16 * ((l16 >> 2) & 1), vrun = 16 * (g & 1), mine = vrun + 8 * (g >> 1);
  const int32_t* table = c.table + int64_t(i) * c.width;
  // without a window the first step is known before the lengths are: its pages are on their way with them
  const int guess = (split * p.span + wave * NS) * kStep;
  int kentry[NS], ventry[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    kentry[n] = table[min((guess + n * kStep + krun) >> shift_b, c.width - 1)];
    ventry[n] = table[min((guess + n * kStep + vrun) >> shift_b, c.width - 1)];
  }
  const Reach r = reach_of(c, a, i, p.rep, first, kTile);
  if (first >= r.rows || r.rows > p.few_rows) return;
  const int c0 = r.lo / kStep, c1 = max(c0, (r.hi + kStep - 1) / kStep), used = max(1, (c1 - c0 + p.span - 1) / p.span);
  if (split >= used) return;
  const int begin = c0 + split * p.span, end = min(c1, begin + p.span);

  // the lane's row
  const int R = first + l16;
  const bool live = R < r.rows;
  const int pos = r.pos0 + R / p.rep, khi = live ? key_end(a, r.len, pos) : 0, klo = live ? key_begin(a, pos) : 0;
  // keys that all rows reach
  const int last = min(first + kTile, r.rows) - 1, all_lo = key_begin(a, r.pos0 + last / p.rep), all_hi = key_end(a, r.len, r.pos0 + first / p.rep);

  auto known = [&](int key, int entry) { return key < r.len && entry >= 0 && entry < c.pages ? entry : -1; };
  auto page_at = [&](int key) { return known(key, table[min(key >> shift_b, c.width - 1)]); };
  int koff[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) koff[b] = 64 * b + 16 * g < d ? 64 * b + 16 * g : 0;    // behind the channels: anything, q is zero there
  uint4 kc[NS][2][DB], vc[NS][kPairs];
  int step = begin + wave * NS, kp[NS], vp[NS];
  float ks[NS], vs[NS];
  // the steps' codes of k, and their scales
  auto load_k = [&](int at) {
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int key = (at + n) * kStep + krun;
      const int8_t* base = c.k + ((int64_t(max(kp[n], 0)) * c.heads + head) * B + (key & (B - 1)) + 8 * (l16 >> 3) + (l16 & 3)) * d;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int b = 0; b < DB; ++b) kc[n][t][b] = *reinterpret_cast<const uint4*>(base + 4 * t * d + koff[b]);
    }
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int64_t s = int64_t(max(vp[n], 0)) * c.heads + head;
      ks[n] = c.kscale[s];
      vs[n] = c.vscale[s];
    }
  };
  if (step < end) {
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int key = (step + n) * kStep;
      kp[n] = c0 == 0 ? known(key + krun, kentry[n]) : page_at(key + krun);
      vp[n] = c0 == 0 ? known(key + vrun, ventry[n]) : page_at(key + vrun);
    }
    load_k(step);
  }

  // half a wave a row, eight channels a lane
  for (int rr = tid >> 5; rr < kTile; rr += kThreads / 32) {
    const int chunk = tid & 31, RR = first + rr, tok = RR / p.rep;
    float v[8];
    uint32_t bits = 0;
    const bool in = RR < r.rows && 8 * chunk < d;
    const elem* x = static_cast<const elem*>(a.q) + int64_t(r.row0 + (in ? tok : 0)) * a.ldq + int64_t(head * p.rep + (in ? RR - tok * p.rep : 0)) * a.hsq +
                    (in ? 8 * chunk : 0);
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 f = load4(x + e);
      v[e] = in ? f.x : 0.f; v[e + 1] = in ? f.y : 0.f; v[e + 2] = in ? f.z : 0.f; v[e + 3] = in ? f.w : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) bits = max(bits, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) bits = max(bits, uint32_t(__shfl_xor(int(bits), m)));
    const QueryScale qs = query_scale(bits, a);
    half8_t h, rest;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float f0 = v[j] * qs.up, f1 = v[j + 1] * qs.up;
      const half2_t x2 = to_half(f0, f1);
      h[j] = x2[0];
      h[j + 1] = x2[1];
      if constexpr (kF32) {
        const half2_t y2 = to_half(f0 - float(x2[0]), f1 - float(x2[1]));
        rest[j] = y2[0];
        rest[j + 1] = y2[1];
      }
    }
    if (chunk < 8 * DB) {
      const int at = ((chunk >> 3) * 2 + (chunk & 1)) * 64 + ((chunk >> 1) & 3) * 16 + rr;
      q_lds[at] = h;
      if constexpr (kF32) q_lds[DB * 2 * 64 + at] = rest;
    }
    if (chunk == 0) unit_lds[rr] = qs.unit;
  }
  __syncthreads();
  const float unit = unit_lds[l16];

  f32x4_t o[2 * kPairs];
#pragma unroll
  for (int m = 0; m < 2 * kPairs; ++m) o[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float M = kNoKey, l = 0.f, mz = kNoKey, lz = 0.f;      // mz, lz: keys whose page of v is zeros
  bool based = false;                                    // whether a row of the wave has a reference

  for (; step < end; step += kWaves * NS) {
    const int key0 = step * kStep, next = step + kWaves * NS;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int8_t* base = c.v + (int64_t(max(vp[n], 0)) * c.heads + head) * d * B + ((key0 + n * kStep + vrun) & (B - 1));
#pragma unroll
      for (int m = 0; m < kPairs; ++m)      // a last half pair: any channels, they are not written
        if (EXACT || 32 * m < d)
          vc[n][m] = *reinterpret_cast<const uint4*>(base + (EXACT ? 32 * m + 16 * (g >> 1) : min(32 * m + 16 * (g >> 1), d - 16)) * B + l16 * B);
    }
    // what becomes of the lane's eight keys of each step: those of [from, to) count
    ValueScale s[NS];
    float f[NS];         // x f: the score in log2
    int from[NS], to[NS];
    bool odd = key0 < all_lo || key0 + kKeys > all_hi || step + NS > end;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      s[n] = value_scale(vs[n]);
      f[n] = unit * ks[n];
      const int at = key0 + n * kStep + mine;
      from[n] = vp[n] < 0 || step + n >= end ? 8 : klo - at;
      to[n] = khi - at;
      odd |= __ballot(vp[n] < 0 || s[n].zero) != 0;
    }
    if (next < end) {
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        kp[n] = page_at((next + n) * kStep + krun);
        vp[n] = page_at((next + n) * kStep + vrun);
      }
    }
    f32x4_t x[NS][2];
#pragma unroll
    for (int n = 0; n < NS; ++n) x[n][0] = x[n][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < DB; ++b) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        half8_t q[kParts];
#pragma unroll
        for (int e = 0; e < kParts; ++e) q[e] = q_lds[((e * DB + b) * 2 + h) * 64 + lane];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const uint4 &ka = kc[n][0][b], &kb = kc[n][1][b];
          const half8_t k0 = h ? half_codes(ka.z, ka.w) : half_codes(ka.x, ka.y), k1 = h ? half_codes(kb.z, kb.w) : half_codes(kb.x, kb.y);
#pragma unroll
          for (int e = kParts - 1; e >= 0; --e) {
            x[n][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[e], x[n][0], 0, 0, 0);
            x[n][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[e], x[n][1], 0, 0, 0);
          }
        }
      }
    }
    if (next < end) load_k(next);
    bool far = p.cap == kCapWide;      // whether scores may be large, or take the cap of large ones
#pragma unroll
    for (int n = 0; n < NS; ++n) far |= f[n] > near_factor(DB);
    if (p.cap == kCapNear) {
      far &= p.cap_out > kFar;
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const float in = f[n] * p.cap_in;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[n][e >> 2][e & 3] = capped<kF32>(x[n][e >> 2][e & 3] * in, p.cap_out);
        f[n] = 1.f;
      }
    }
    auto in = [&](int n, int e) { return bool(int(e >= from[n]) & int(e < to[n]) & int(!s[n].zero)); };
    far = __ballot(far) != 0;
    odd |= based || far;
    float top = kNoKey;
    if (!odd) {
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        float t = kNoKey;
#pragma unroll
        for (int e = 0; e < 8; ++e) t = fmaxf(t, x[n][e >> 2][e & 3] * f[n]);
        top = fmaxf(top, t + s[n].exp);
      }
    } else {
      if (p.cap == kCapWide) {
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          const float in = f[n] * p.cap_in;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[n][e >> 2][e & 3] = capped_wide(x[n][e >> 2][e & 3] * in, p.cap_out);
          f[n] = 1.f;
        }
      }
      if (based || far) {
        float most = kNoKey;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) most = in(n, e) ? fmaxf(most, x[n][e >> 2][e & 3] * f[n]) : most;
        const float old = based ? base_lds[wave * kTile + l16] : 0.f, base = next_base(across(most), old, M == kNoKey);
        M = M == kNoKey ? M : M + (old - base);
        based = __ballot(base != 0.f) != 0;
        if (based) base_lds[wave * kTile + l16] = base;
        if (base != 0.f) {
#pragma unroll
          for (int n = 0; n < NS; ++n) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[n][e >> 2][e & 3] = x[n][e >> 2][e & 3] * f[n] - (s[n].zero ? 0.f : base);
            f[n] = 1.f;
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        float t = kNoKey;
#pragma unroll
        for (int e = 0; e < 8; ++e) t = int(e >= from[n]) & int(e < to[n]) ? fmaxf(t, x[n][e >> 2][e & 3] * f[n]) : t;
        if (__ballot(s[n].zero)) {
          // keys of pages of zeros count in the sum of weights only, on a maximum of their own
          const float now = fmaxf(mz, across(s[n].zero ? t : kNoKey));
          lz *= __builtin_amdgcn_exp2f(mz - now);
          mz = now;
          if (s[n].zero) {
#pragma unroll
            for (int e = 0; e < 8; ++e) lz += int(e >= from[n]) & int(e < to[n]) ? __builtin_amdgcn_exp2f(x[n][e >> 2][e & 3] * f[n] - now) : 0.f;
          }
        }
        top = s[n].zero || t == kNoKey ? top : fmaxf(top, t + s[n].exp);
      }
    }
    const float now = fmaxf(M, ceilf(across(top)) - kTop);
    if (__ballot(now != M)) {
      const float back = __builtin_amdgcn_exp2f(M - now);
      l *= back;
#pragma unroll
      for (int m = 0; m < 2 * kPairs; ++m) o[m] *= back;
      M = now;
    }
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const float shift = s[n].exp - M;
      float P[8], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) P[e] = __builtin_amdgcn_exp2f(fmaf(x[n][e >> 2][e & 3], f[n], shift));
      if (odd) {
#pragma unroll
        for (int e = 0; e < 8; ++e) P[e] = in(n, e) ? P[e] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum += P[e];
        P[e] *= s[n].mant;
      }
      if (odd) {      // a scale that is no number must not reach keys that do not count
#pragma unroll
        for (int e = 0; e < 8; ++e) P[e] = in(n, e) ? P[e] : 0.f;
      }
      half8_t w[kParts];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const half2_t h = to_half(P[e], P[e + 1]);
        w[0][e] = h[0];
        w[0][e + 1] = h[1];
        if constexpr (kF32) {
          const half2_t rest = to_half(P[e] - float(h[0]), P[e + 1] - float(h[1]));
          w[1][e] = rest[0];
          w[1][e + 1] = rest[1];
        }
      }
      l += sum * s[n].inv;
#pragma unroll
      for (int m = 0; m < kPairs; ++m) {
        if (!EXACT && 32 * m >= d) continue;
        const uint4& v = vc[n][m];
        const auto lo = __builtin_amdgcn_permlane32_swap(v.x, v.z, false, false), hi = __builtin_amdgcn_permlane32_swap(v.y, v.w, false, false);
        const half8_t v0 = half_codes(lo[0], hi[0]), v1 = half_codes(lo[1], hi[1]);
#pragma unroll
        for (int e = kParts - 1; e >= 0; --e) {
          o[2 * m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[e], o[2 * m], 0, 0, 0);
          o[2 * m + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[e], o[2 * m + 1], 0, 0, 0);
        }
      }
    }
  }

  // the wave's sums, then the waves'
  l = sum_across(l);
  lz = sum_across(lz);
  const Finish fin = finish_of(M, based ? base_lds[wave * kTile + l16] : 0.f);
  const float both = fmaxf(fin.all, mz);
  l = l * (fin.sum_unit * __builtin_amdgcn_exp2f(fin.all - both)) + lz * __builtin_amdgcn_exp2f(mz - both);
  if (g == 0) *reinterpret_cast<float2*>(sum_lds + 2 * (wave * kTile + l16)) = make_float2(both, l);
  __syncthreads();
  float top = kNoKey;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sum_lds[2 * (w * kTile + l16)]);
  const float mul = fin.unit * __builtin_amdgcn_exp2f(fin.all - top);
  if (l16 < p.keep) {
    float* at = out_lds + (wave * p.keep + l16) * ld + 4 * g;
#pragma unroll
    for (int m = 0; m < 2 * kPairs; ++m)
      if (EXACT || 16 * m < d) *reinterpret_cast<f32x4_t*>(at + 16 * m) = o[m] * mul;
  }
  __syncthreads();
  const int per = d / 4;
  const int64_t part = (int64_t(i) * p.splits + split) * gridDim.x + blockIdx.x;
  for (int e = tid; e < p.keep * per; e += kThreads) {
    const int row = e / per, ch = e % per * 4, RR = first + row;
    if (RR >= r.rows) break;
    float big = kNoKey, total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) big = fmaxf(big, sum_lds[2 * (w * kTile + row)]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sum_lds[2 * (w * kTile + row) + 1] * __builtin_amdgcn_exp2f(sum_lds[2 * (w * kTile + row)] - big);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += *reinterpret_cast<const f32x4_t*>(out_lds + (w * p.keep + row) * ld + ch);
    if (used > 1) {
      *reinterpret_cast<f32x4_t*>(p.parts + (part * p.keep + row) * d + ch) = v;
      if (ch == 0) *reinterpret_cast<float2*>(p.sums + 2 * (part * p.keep + row)) = make_float2(big, total);
    } else {
      store_row<Tag>(p, r, RR, head, ch, v, big, total);
    }
  }
}

// The parts of a row's keys joined: a workgroup a row, groups of d / 4 threads take the parts in turn and are added in order.
template <class Tag>
__global__ __launch_bounds__(kJoin) void attend_join_kernel(const AttendPlan p) {
  __shared__ f32x4_t group_lds[kJoin];
  __shared__ float2 sum_lds[kJoin];
  const cafeq_cache& c = p.c;
  const int i = blockIdx.y, x = blockIdx.x, tile = p.tiles == 1 ? 0 : x / c.heads, head = x - tile * c.heads, d = c.d, first = tile * kTile;
  const int row = blockIdx.z, tid = threadIdx.x;
  const Reach r = reach_of(c, p.a, i, p.rep, first, kTile);
  const int c0 = r.lo / kStep, c1 = max(c0, (r.hi + kStep - 1) / kStep), used = (c1 - c0 + p.span - 1) / p.span;
  if (first + row >= r.rows || r.rows > p.few_rows || used <= 1) return;
  const int per = d / 4, groups = kJoin / per, group = tid / per, ch = (tid - group * per) * 4;
  const int64_t part = (int64_t(i) * p.splits * gridDim.x + x) * p.keep + row, step = int64_t(gridDim.x) * p.keep;
  // the largest M; then weights and values in units of it
  float big = kNoKey;
  for (int s = tid; s < used; s += kJoin) big = fmaxf(big, p.sums[2 * (part + s * step)]);
  for (int m = 1; m < 64; m <<= 1) big = fmaxf(big, __shfl_xor(big, m));
  if ((tid & 63) == 0) sum_lds[tid >> 6].x = big;
  __syncthreads();
  for (int w = 0; w < kJoin / 64; ++w) big = fmaxf(big, sum_lds[w].x);
  float total = 0.f;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (group < groups) {
#pragma unroll 4
    for (int s = group; s < used; s += groups) {
      const int64_t at = part + s * step;
      const float2 m = *reinterpret_cast<const float2*>(p.sums + 2 * at);
      const float w = __builtin_amdgcn_exp2f(m.x - big);
      total += m.y * w;
      v += *reinterpret_cast<const f32x4_t*>(p.parts + at * d + ch) * w;
    }
  }
  __syncthreads();
  group_lds[tid] = v;
  sum_lds[tid].y = total;
  __syncthreads();
  if (group != 0) return;
  for (int k = 1; k < groups; ++k) {
    v += group_lds[k * per + tid];
    total += sum_lds[k * per + tid].y;
  }
  store_row<Tag>(p, r, first + row, head, ch, v, big, total);
}

template <class Tag, int DB, bool EXACT>
int launch(const AttendPlan& p, hipStream_t st) {
  // Workgroups go round the eight XCDs in turn: with the heads innermost, each sequence's keys are spread over all of them however long it is.
  // 48 sequences of 1600 to 32700 keys, 16 heads of 128, sequences innermost: 842 us, heads innermost 629.
  const dim3 grid(unsigned(p.c.heads * p.tiles), unsigned(p.splits), unsigned(p.c.sequences));
  const int parts = Tag::dtype == CAFEQ_F32 ? 2 : 1;
  const size_t lds = sizeof(float) * (parts * DB * 2 * 64 * 4 + kTile + kWaves * kTile * 3 + size_t(kWaves) * p.keep * (p.c.d + 4));
  const auto kern = attend_few_kernel<Tag, DB, EXACT>;
  if (lds > 65536) {
    static const bool ok = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess;
    if (!ok) return CAFEQ_ERR_LAUNCH;
  }
  hipLaunchKernelGGL(kern, grid, dim3(kThreads), lds, st, p);
  CAFEQ_CHECK_LAUNCH();
  if (p.splits > 1) {
    hipLaunchKernelGGL((attend_join_kernel<Tag>), dim3(grid.x, grid.z, unsigned(p.keep)), dim3(kJoin), 0, st, p);
    CAFEQ_CHECK_LAUNCH();
  }
  return CAFEQ_OK;
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

int launch_attend_few(const AttendPlan& p, hipStream_t st) {
  return p.a.dtype == CAFEQ_F32 ? launch_type<F32Tag>(p, st) : launch_type<BF16Tag>(p, st);
}

}  // namespace cafeq
