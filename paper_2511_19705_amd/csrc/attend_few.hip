// Attention of few new tokens a sequence over the 8-bit cache: memory is the bound, so everything serves the loads.
#include "attend.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kTile = 16, kStep = 64;

__device__ __forceinline__ float across(float v) {      // largest over the four lanes of a row
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_across(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A workgroup: 16 rows (tokens and query heads that share a key head) over a part of the keys; its waves take steps of 64 keys in turn and
// join in the end.  Lanes l % 16 hold a row, g = l / 16 the keys 16 g .. 16 g + 15 of a step: tile t of the first product, v_mfma 16x16x32,
// has key 16 (r / 4) + 4 t + r % 4 in row r, so that a lane's four results of four tiles are the 16 keys whose codes of v lie side by side in
// its 16 bytes.  Codes go from memory to registers, the next step's of k while this one is worked on.
template <class Tag, int DB>
__global__ __launch_bounds__(kThreads) void attend_few_kernel(const AttendPlan p) {
  using elem = typename Tag::elem;
  constexpr bool kF32 = Tag::dtype == CAFEQ_F32;
  constexpr int kParts = kF32 ? 2 : 1, kLd = 64 * DB + 4;
  __shared__ float sum_lds[kWaves][kTile][2];
  __shared__ float out_lds[kWaves][kTile][kLd];
  const cafeq_cache& c = p.c;
  const cafeq_attention& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.y, split = blockIdx.x % p.splits, tile = blockIdx.x / p.splits % p.tiles, i = blockIdx.x / p.splits / p.tiles;
  const int d = c.d, B = c.block, first = tile * kTile;
  const Reach r = reach_of(c, a, i, p.rep, first, kTile);
  if (first >= r.rows) return;
  const int c0 = r.lo / kStep, c1 = max(c0, (r.hi + kStep - 1) / kStep), used = max(1, (c1 - c0 + p.span - 1) / p.span);
  if (split >= used) return;
  const int begin = c0 + split * p.span, end = min(c1, begin + p.span);

  // the lane's row
  const int R = first + l16, token = R / p.rep, qhead = head * p.rep + R % p.rep;
  const bool live = R < r.rows;
  const int pos = r.pos0 + token, khi = live ? key_end(a, r.len, pos) : 0, klo = live ? key_begin(a, pos) : 0;
  // keys that all rows reach
  const int last = min(first + kTile, r.rows) - 1, all_lo = key_begin(a, r.pos0 + last / p.rep), all_hi = key_end(a, r.len, r.pos0 + first / p.rep);

  half8_t q[kParts][DB][2];
  float unit;          // a product's sum times this, times the scale of k, is the score (in log2 without a soft cap)
  {
    float v[DB][16], top = 0.f;
    uint32_t bits = 0;
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const int ch = 64 * b + 16 * g;
      const elem* x = static_cast<const elem*>(a.q) + int64_t(r.row0 + token) * a.ldq + int64_t(qhead) * a.hsq + ch;
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const float4 f = live && ch < d ? load4(x + e) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[b][e] = f.x; v[b][e + 1] = f.y; v[b][e + 2] = f.z; v[b][e + 3] = f.w;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        top = fmaxf(top, fabsf(v[b][e]));
        bits = max(bits, __float_as_uint(v[b][e]) & 0x7FFFFFFFu);
      }
    }
    top = across(top);
    bits = max(bits, uint32_t(__shfl_xor(int(bits), 16)));
    bits = max(bits, uint32_t(__shfl_xor(int(bits), 32)));
    // the row's largest magnitude to [2^14, 2^15): bfloat16 then is exact in float16 down to 2^-28 of it
    const int e = max(-100, int(bits >> 23) - 127);
    const float up = bits ? ldexpf(1.f, 14 - e) : 1.f;
    unit = bits ? ldexpf(a.scale, e - 14) : 0.f;
    if (bits >= 0x7F800000u) unit = NAN;
    if (a.softcap <= 0.f) unit *= kLog2e;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float f = v[b][8 * s + j] * up;
          q[0][b][s][j] = _Float16(f);
          if constexpr (kF32) q[1][b][s][j] = _Float16(f - float(q[0][b][s][j]));
        }
  }

  int koff[DB];
#pragma unroll
  for (int b = 0; b < DB; ++b) koff[b] = 64 * b + 16 * g < d ? 64 * b + 16 * g : 0;    // behind the channels: anything, q is zero there
  const int krun = 16 * (l16 >> 2), vrun = 16 * g;
  uint4 kc[4][DB], vc[4 * DB];
  auto page_at = [&](int key) { return key < r.len ? page_of(c, i, key / B) : -1; };
  auto load_k = [&](int step, int page) {
    const int key = step * kStep + krun;
    const int8_t* base = c.k + ((int64_t(max(page, 0)) * c.heads + head) * B + (key & (B - 1)) + (l16 & 3)) * d;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < DB; ++b) kc[t][b] = *reinterpret_cast<const uint4*>(base + 4 * t * d + koff[b]);
  };

  f32x4_t o[4 * DB];
#pragma unroll
  for (int m = 0; m < 4 * DB; ++m) o[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float M = kNoKey, l = 0.f, mz = kNoKey, lz = 0.f;      // mz, lz: keys whose page of v is zeros

  int step = begin + wave, kp = -1, vp = -1;
  float ks = 0.f, vs = 0.f;
  auto scales = [&](int page) {
    const int64_t at = int64_t(max(page, 0)) * c.heads + head;
    ks = c.kscale[at];
    vs = c.vscale[at];
  };
  if (step < end) {
    kp = page_at(step * kStep + krun);
    vp = page_at(step * kStep + vrun);
    load_k(step, kp);
    scales(vp);
  }
  for (; step < end; step += kWaves) {
    const int key0 = step * kStep, next = step + kWaves;
    {
      const int8_t* base = c.v + ((int64_t(max(vp, 0)) * c.heads + head) * d + l16) * B + ((key0 + vrun) & (B - 1));
#pragma unroll
      for (int m = 0; m < 4 * DB; ++m)
        if (16 * m < d) vc[m] = *reinterpret_cast<const uint4*>(base + int64_t(16 * m) * B);
    }
    const bool whole = key0 >= all_lo && key0 + kStep <= all_hi && __ballot(vp < 0) == 0;
    const int page = vp;
    const float ck = unit * ks;
    const ValueScale s = value_scale(vs);
    if (next < end) {
      kp = page_at(next * kStep + krun);
      vp = page_at(next * kStep + vrun);
    }
    f32x4_t x[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      x[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const half8_t k0 = half_codes(kc[t][b].x, kc[t][b].y), k1 = half_codes(kc[t][b].z, kc[t][b].w);
#pragma unroll
        for (int e = kParts - 1; e >= 0; --e) {
          x[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[e][b][0], x[t], 0, 0, 0);
          x[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[e][b][1], x[t], 0, 0, 0);
        }
      }
    }
    if (next < end) {
      load_k(next, kp);
      scales(vp);
    }
    float f = ck;        // x f: the score in log2
    if (a.softcap > 0.f) {
      const float in = ck / a.softcap, out = a.softcap * kLog2e;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float z = x[t][j] * in;
          if constexpr (kF32) x[t][j] = tanhf(z) * out;
          else x[t][j] = out - 2.f * out * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * kLog2e * z));
        }
      f = 1.f;
    }
    bool in[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = key0 + vrun + e;
      in[e] = whole || (page >= 0 && key >= klo && key < khi);
    }
    const bool zeros = s.zero;
    float top = kNoKey;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = in[e] ? fmaxf(top, x[e >> 2][e & 3] * f) : top;
    if (__ballot(zeros)) {
      // keys of pages of zeros count in the sum of weights only, on a maximum of their own
      const float mine = across(zeros ? top : kNoKey), now = fmaxf(mz, mine);
      lz *= __builtin_amdgcn_exp2f(mz - now);
      mz = now;
      if (zeros) {
#pragma unroll
        for (int e = 0; e < 16; ++e) lz += in[e] ? __builtin_amdgcn_exp2f(x[e >> 2][e & 3] * f - now) : 0.f;
      }
    }
    const float now = fmaxf(M, ceilf(across(zeros || top == kNoKey ? kNoKey : top + s.exp)) - kTop);
    if (__ballot(now != M)) {
      const float back = __builtin_amdgcn_exp2f(M - now);
      l *= back;
#pragma unroll
      for (int m = 0; m < 4 * DB; ++m) o[m] *= back;
      M = now;
    }
    const float shift = s.exp - M;
    half8_t w[kParts][2];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const bool some = in[e] && !zeros;        // (a scale that is no number must not reach keys that do not count)
      const float P = some ? __builtin_amdgcn_exp2f(fmaf(x[e >> 2][e & 3], f, shift)) : 0.f;
      sum += P;
      const float weight = some ? P * s.mant : 0.f;
      const _Float16 h = _Float16(weight);
      w[0][e >> 3][e & 7] = h;
      if constexpr (kF32) w[1][e >> 3][e & 7] = _Float16(weight - float(h));
    }
    l += sum * s.inv;
#pragma unroll
    for (int m = 0; m < 4 * DB; ++m) {
      if (16 * m >= d) continue;
      const half8_t v0 = half_codes(vc[m].x, vc[m].y), v1 = half_codes(vc[m].z, vc[m].w);
#pragma unroll
      for (int e = kParts - 1; e >= 0; --e) {
        o[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w[e][0], o[m], 0, 0, 0);
        o[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w[e][1], o[m], 0, 0, 0);
      }
    }
  }

  // the wave's sums, then the waves'
  l = sum_across(l);
  lz = sum_across(lz);
  const float both = fmaxf(M, mz), own = __builtin_amdgcn_exp2f(M - both);
  l = l * own + lz * __builtin_amdgcn_exp2f(mz - both);
  if (g == 0) {
    sum_lds[wave][l16][0] = both;
    sum_lds[wave][l16][1] = l;
  }
  __syncthreads();
  float top = kNoKey;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sum_lds[w][l16][0]);
  const float mul = __builtin_amdgcn_exp2f(M - top);
#pragma unroll
  for (int m = 0; m < 4 * DB; ++m) *reinterpret_cast<f32x4_t*>(&out_lds[wave][l16][16 * m + 4 * g]) = o[m] * mul;
  __syncthreads();
  const int per = d / 4;
  const int64_t part = (int64_t(i * p.tiles + tile) * c.heads + head) * p.splits + split;
  for (int e = tid; e < kTile * per; e += kThreads) {
    const int row = e / per, ch = e % per * 4, RR = first + row;
    if (RR >= r.rows) break;
    float big = kNoKey, total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) big = fmaxf(big, sum_lds[w][row][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += sum_lds[w][row][1] * __builtin_amdgcn_exp2f(sum_lds[w][row][0] - big);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += *reinterpret_cast<const f32x4_t*>(&out_lds[w][row][ch]);
    if (used > 1) {
      *reinterpret_cast<f32x4_t*>(p.parts + (part * p.keep + row) * d + ch) = v;
      if (ch == 0) *reinterpret_cast<float2*>(p.sums + 2 * (part * p.keep + row)) = make_float2(big, total);
    } else {
      store_row<Tag>(p, r, RR, head, ch, v, big, total);
    }
  }
}

// Parts of a tile's keys joined in their order.
template <class Tag>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(const AttendPlan p) {
  const cafeq_cache& c = p.c;
  const int head = blockIdx.y, tile = blockIdx.x % p.tiles, i = blockIdx.x / p.tiles, d = c.d, first = tile * kTile;
  const Reach r = reach_of(c, p.a, i, p.rep, first, kTile);
  const int c0 = r.lo / kStep, c1 = max(c0, (r.hi + kStep - 1) / kStep), used = (c1 - c0 + p.span - 1) / p.span;
  if (first >= r.rows || used <= 1) return;
  const int per = d / 4;
  const int64_t part = (int64_t(i * p.tiles + tile) * c.heads + head) * p.splits;
  for (int e = threadIdx.x; e < kTile * per; e += kThreads) {
    const int row = e / per, ch = e % per * 4;
    if (first + row >= r.rows) break;
    float big = kNoKey, total = 0.f;
    for (int s = 0; s < used; ++s) big = fmaxf(big, p.sums[2 * ((part + s) * p.keep + row)]);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < used; ++s) {
      const int64_t at = (part + s) * p.keep + row;
      const float2 m = *reinterpret_cast<const float2*>(p.sums + 2 * at);
      const float w = __builtin_amdgcn_exp2f(m.x - big);
      total += m.y * w;
      v += *reinterpret_cast<const f32x4_t*>(p.parts + at * d + ch) * w;
    }
    store_row<Tag>(p, r, first + row, head, ch, v, big, total);
  }
}

template <class Tag>
int launch_type(const AttendPlan& p, hipStream_t st) {
  const dim3 grid(unsigned(int64_t(p.c.sequences) * p.tiles * p.splits), unsigned(p.c.heads)), block(kThreads);
  switch ((p.c.d + 63) / 64) {
    case 1: hipLaunchKernelGGL((attend_few_kernel<Tag, 1>), grid, block, 0, st, p); break;
    case 2: hipLaunchKernelGGL((attend_few_kernel<Tag, 2>), grid, block, 0, st, p); break;
    case 3: hipLaunchKernelGGL((attend_few_kernel<Tag, 3>), grid, block, 0, st, p); break;
    default: hipLaunchKernelGGL((attend_few_kernel<Tag, 4>), grid, block, 0, st, p); break;
  }
  CAFEQ_CHECK_LAUNCH();
  if (p.splits > 1) {
    hipLaunchKernelGGL((attend_join_kernel<Tag>), dim3(unsigned(int64_t(p.c.sequences) * p.tiles), unsigned(p.c.heads)), block, 0, st, p);
    CAFEQ_CHECK_LAUNCH();
  }
  return CAFEQ_OK;
}

}  // namespace

int launch_attend_few(const AttendPlan& p, hipStream_t st) {
  return p.a.dtype == CAFEQ_F32 ? launch_type<F32Tag>(p, st) : launch_type<BF16Tag>(p, st);
}

}  // namespace cafeq
