// Products with packed 4-bit weights for many tokens: tiles on the 32x32 matrix instructions.
//   y[t][o] = sum over units of s[o][unit] (sx[t][unit]) sum_{c in unit} q[o][c] x[t][c]
// A workgroup of four waves owns 32 MT tokens x 256 rows of the weight; a wave owns all its tokens and 64 of the rows.  The
// activations of 128 columns go to LDS asynchronously, a stage ahead of the one being multiplied; the weights, which no other
// wave of the workgroup needs, go to registers, 4 bits a weight, and are unpacked there once for the 32 MT tokens.
#include "cafeq_common.hpp"
#include "cafeq_internal.hpp"
#include "packed.hpp"

namespace cafeq {
namespace {

using i32x16 = __attribute__((__vector_size__(16 * sizeof(int)))) int;
using f32x16 = __attribute__((__vector_size__(16 * sizeof(float)))) float;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kWaveRows = 64, kTileRows = kWaves * kWaveRows;

struct GemmArgs {
  const uint8_t* packed;
  PackedShape p;
  const uint8_t* x;       // [planes][n][ldx]
  int64_t ldx;            // bytes
  int64_t plane;          // bytes from a plane to the next
  int planes;
  const float* xscales;   // [n][xgroups]
  int64_t xgroups;
  int wunits, xunits;     // units a scale
  int64_t n;
  void* y;
  int64_t ldy;
  int ydtype;
  int tok_tiles, row_tiles;  // tiles of the workgroups
  int whole;              // tiles that one workgroup takes whole; of the others every one goes to `split` of them
  int split;
  float* part;            // [tile - whole][split][32 MT * 256], in the accumulators' order
};

// tile number -> (token tile, row tile): token tiles of a group of eight side by side, so that workgroups that run together share
// activations and weights in their L2
__device__ __forceinline__ void place(int id, const GemmArgs& a, int* tt, int* rt) {
  const int per = 8 * a.row_tiles, g = id / per, in = id % per;
  const int size = min(8, a.tok_tiles - 8 * g);
  *tt = 8 * g + in % size;
  *rt = in / size;
}

// The matrix instructions over 128 columns; lane l of an operand holds row (or token) l % 32, lane half h = l / 32
template <bool I8> struct Form;
template <> struct Form<true> {
  using Frag = i32x4;
  static constexpr int kRowBytes = 128;   // a token's 128 columns
  static constexpr int kSteps = 4;        // instructions: 32 columns each, half h their 16 h + 0 .. 15
  // q0, q1: the row's chunks h and h + 2, each with 16 columns of either 64
  static __device__ __forceinline__ void unpack(Frag (&b)[kSteps], const uint4& q0, const uint4& q1) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const uint4& q = i & 1 ? q1 : q0;
      const uint32_t d0 = i < 2 ? q.x : q.z, d1 = i < 2 ? q.y : q.w;
      b[i] = i32x4{int(low16(d0)), int(high16(d0)), int(low16(d1)), int(high16(d1))};
    }
  }
};
template <> struct Form<false> {
  using Frag = bf16x8_t;
  static constexpr int kRowBytes = 256;
  static constexpr int kSteps = 8;        // 16 columns each: of block i / 2 of 32, half h its 16 h + 8 (i % 2) + 0 .. 7
  static __device__ __forceinline__ void unpack(Frag (&b)[kSteps], const uint4& q0, const uint4& q1) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const uint4& q = i >> 1 & 1 ? q1 : q0;
      b[i] = bf16_codes(i < 4 ? (i & 1 ? q.y : q.x) : (i & 1 ? q.w : q.z));
    }
  }
};

template <bool I8, int MT, int FG, bool SX>
__global__ __launch_bounds__(kThreads, 2) void packed_gemm_kernel(const GemmArgs a) {
  using F = Form<I8>;
  constexpr int NT = 2, ROWB = F::kRowBytes, CH = ROWB / 16, SLOT = 32 * MT * ROWB;
  constexpr int NDMA = SLOT / 16 / kThreads;        // requests of a thread and stage
  constexpr int UPB = kBlockK / FG, SPU = F::kSteps / UPB;
  constexpr int TOK = 32 * MT;
  extern __shared__ __align__(16) unsigned char smem[];   // [2][TOK][ROWB], then [2][UPB][TOK] scales of the activations
  const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // which tile, which of its stages
  const int nkb = int(a.p.kblocks), stages = nkb * a.planes;
  int id = blockIdx.x, s0 = 0, s1 = stages, piece = -1;
  // whole tiles, and pieces, that are neighbours behind one L2 (workgroups go round the eight XCDs in turn)
  auto near = [](int i, int total) { return (total & 7) == 0 ? (i & 7) * (total >> 3) + (i >> 3) : i; };
  if (id < a.whole) {
    id = near(id, a.whole);
  } else {
    piece = near(id - a.whole, gridDim.x - a.whole);
    const int k = piece % a.split;
    id = a.whole + piece / a.split;
    s0 = int(int64_t(stages) * k / a.split);
    s1 = int(int64_t(stages) * (k + 1) / a.split);
  }
  int tt, rt;
  place(id, a, &tt, &rt);
  const int64_t t0 = int64_t(tt) * TOK;
  const int last = int(min(int64_t(TOK), a.n - t0)) - 1;          // last token of the tile
  const int64_t row0 = int64_t(rt) * kTileRows + wave * kWaveRows; // the wave's first row

  // Requests of the activations: a thread's piece i is 16 bytes of token row i * RSTEP + tid / CH (past the last one: that one's).
  // The chunks of a token lie in LDS at their number XOR the token, so that the operand reads of eight tokens fall on distinct
  // banks.  (Opaque to the compiler, which would otherwise drain every request before each LDS read; the address assumes
  // that dynamic LDS starts at 0.)
  constexpr int RSTEP = kThreads / CH;
  const uint32_t ldx = uint32_t(a.ldx), rmax = uint32_t(last) * ldx, rfirst = uint32_t(tid / CH) * ldx;
  const uint32_t ch = uint32_t((tid % CH) ^ (tid / CH & 7)) * 16u;
  const uint32_t tail = uint32_t(a.p.cols - int64_t(nkb - 1) * kBlockK) * (ROWB / kBlockK);   // bytes of a token in the last block
  const uint8_t* xbase = a.x + t0 * a.ldx;
  auto dma = [&](int plane, int kb, int slot) __attribute__((always_inline)) {
    const uint8_t* src = xbase + plane * a.plane + int64_t(kb) * ROWB;
    const uint32_t in = kb == nkb - 1 && ch >= tail ? 0u : ch;
    const uint32_t to = uint32_t(slot * SLOT) + uint32_t(wave) * 1024u;
#pragma unroll
    for (int i = 0; i < NDMA; ++i) {
      const uint32_t off = min(rfirst + uint32_t(i * RSTEP) * ldx, rmax) + in;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to + uint32_t(i) * (kThreads * 16u)), "v"(off), "s"(src)
                   : "memory");
    }
  };
  // rows past the matrix read its last tile
  const uint4* wp[NT];
  const float* sp[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int tile = int(min(row0 / kRowTile + 2 * t + (l31 >> 4), a.p.row_tiles - 1));
    wp[t] = reinterpret_cast<const uint4*>(a.packed) + int64_t(tile) * nkb * 64 + h * 16 + (l31 & 15);
    sp[t] = reinterpret_cast<const float*>(a.packed + a.p.scales_at) + int64_t(tile) * a.p.groups * kRowTile + (l31 & 15);
  }
  uint4 wq[NT][2];
  float sw[NT][UPB];
  float sx[SX ? UPB : 1];
  auto load_w = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      wq[t][0] = wp[t][int64_t(kb) * 64];
      wq[t][1] = wp[t][int64_t(kb) * 64 + 32];
#pragma unroll
      for (int u = 0; u < UPB; ++u)
        sw[t][u] = sp[t][min((kb * UPB + u) / a.wunits, int(a.p.groups) - 1) * kRowTile];
    }
    if constexpr (SX) {
      if (tid < TOK)
#pragma unroll
        for (int u = 0; u < UPB; ++u)
          sx[u] = a.xscales[(t0 + min(tid, last)) * a.xgroups + min((kb * UPB + u) / a.xunits, int(a.xgroups) - 1)];
    }
  };

  f32x16 y[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) y[m][t][r] = 0.f;

  int plane = s0 / nkb, kb = s0 % nkb;
  dma(plane, kb, 0);
  load_w(kb);
  for (int s = s0; s < s1; ++s) {
    const int slot = (s - s0) & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this stage's activations and weights
    typename F::Frag b[NT][F::kSteps];
    float sc[NT][UPB];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      F::unpack(b[t], wq[t][0], wq[t][1]);
#pragma unroll
      for (int u = 0; u < UPB; ++u) sc[t][u] = sw[t][u];
    }
    float* xs = reinterpret_cast<float*>(smem + 2 * SLOT) + slot * UPB * TOK;
    if constexpr (SX) {
      if (tid < TOK)
#pragma unroll
        for (int u = 0; u < UPB; ++u) xs[u * TOK + tid] = sx[u];
    }
    __syncthreads();
    if constexpr (!I8) {
      // past the matrix's columns LDS holds others of the token, of which an infinity times a code of zero would be no number
      if (kb == nkb - 1 && tail < uint32_t(ROWB)) {
        if (ch >= tail)
#pragma unroll
          for (int i = 0; i < NDMA; ++i) *reinterpret_cast<uint4*>(smem + slot * SLOT + (i * kThreads + tid) * 16) = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
      }
    }
    if (++kb == nkb) { kb = 0; ++plane; }
    if (s + 1 < s1) {
      dma(plane, kb, slot ^ 1);
      load_w(kb);
    }
    const unsigned char* xt = smem + slot * SLOT + l31 * ROWB;
    const int sz = l31 & 7;
    if constexpr (I8) {
      // Tiles one after another, (token tile, unit, row tile).  While a tile's instructions run, the one before it is taken up in
      // float32: from the second instruction on, when the last one's result is there.
      constexpr int PER = NT * UPB, TILES = MT * PER;
      i32x4 x[4];
      i32x16 acc[2];
      auto read_x = [&](int m, int i) __attribute__((always_inline)) {
        x[i] = *reinterpret_cast<const i32x4*>(xt + m * 32 * ROWB + ((2 * i + h) ^ sz) * 16);
      };
      auto take = [&](int j, int q0, int q1) __attribute__((always_inline)) {
        const int m = j / PER, u = j / NT % UPB, t = j % NT;
#pragma unroll
        for (int q = q0; q < q1; ++q) {
          f32x4 f;
          if constexpr (SX) f = *reinterpret_cast<const f32x4*>(xs + u * TOK + m * 32 + 8 * q + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = float(acc[j & 1][4 * q + e]);
            y[m][t][4 * q + e] = fmaf(SX ? v * f[e] : v, sc[t][u], y[m][t][4 * q + e]);
          }
        }
      };
#pragma unroll
      for (int i = 0; i < 4; ++i) read_x(0, i);
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const int m = j / PER, u = j / NT % UPB, t = j % NT;
#pragma unroll
        for (int i = 0; i < SPU; ++i) {
          acc[j & 1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[u * SPU + i], b[t][u * SPU + i], i == 0 ? i32x16{} : acc[j & 1], 0, 0, 0);
          if (t == NT - 1 && m + 1 < MT) read_x(m + 1, u * SPU + i);
          __builtin_amdgcn_sched_barrier(0);
          if (j > 0) {
            if (SPU == 4) take(j - 1, i == 0 ? 0 : i - 1, i == 0 ? 0 : i == 3 ? 4 : i);
            else if (SPU == 2) take(j - 1, i, i == 0 ? 1 : 4);
            else take(j - 1, 0, 4);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      take(TILES - 1, 0, 4);
    } else {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int u = 0; u < UPB; ++u) {
          f32x16 acc[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t] = f32x16{};
#pragma unroll
          for (int i = u * SPU; i < (u + 1) * SPU; ++i) {
            const bf16x8_t x = *reinterpret_cast<const bf16x8_t*>(xt + m * 32 * ROWB + ((4 * (i >> 1) + 2 * h + (i & 1)) ^ sz) * 16);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, b[t][i], acc[t], 0, 0, 0);
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) y[m][t][r] = fmaf(acc[t][r], sc[t][u], y[m][t][r]);
        }
    }
  }

  if (piece >= 0) {
    float* out = a.part + int64_t(piece) * (TOK * kTileRows) + wave * (MT * NT * 16 * 64) + lane;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[((m * NT + t) * 16 + r) * 64] = y[m][t][r];
    return;
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int tok = m * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
      const float f = (I8 && !SX && tok <= last ? a.xscales[t0 + tok] : 1.f) * 0.0625f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int64_t row = row0 + t * 32 + l31;
        if (tok <= last && row < a.p.rows) store_y(a.y, a.ydtype, (t0 + tok) * a.ldy + row, y[m][t][r] * f);
      }
    }
}

// the pieces of a tile in order, to Y
template <int MT>
__global__ __launch_bounds__(256) void packed_join_kernel(const GemmArgs a, bool per_token) {
  constexpr int N = 32 * MT * kTileRows, NT = 2;
  const int tile = blockIdx.y, e = blockIdx.x * 256 + threadIdx.x;
  int tt, rt;
  place(a.whole + tile, a, &tt, &rt);
  const int lane = e & 63, r = e >> 6 & 15, t = e >> 10 & (NT - 1), m = (e >> 11) % MT, wave = (e >> 11) / MT;
  const int64_t tok = int64_t(tt) * 32 * MT + m * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
  const int64_t row = int64_t(rt) * kTileRows + wave * kWaveRows + t * 32 + (lane & 31);
  if (tok >= a.n || row >= a.p.rows) return;
  const float* p = a.part + int64_t(tile) * a.split * N + e;
  float v = 0.f;
  for (int k = 0; k < a.split; ++k) v += p[int64_t(k) * N];
  store_y(a.y, a.ydtype, tok * a.ldy + row, v * ((per_token ? a.xscales[tok] : 1.f) * 0.0625f));
}

// float32 activations as three planes of bfloat16, the small parts first: hi + mid + lo exactly
__global__ __launch_bounds__(256) void split_planes_of_x_kernel(const float* __restrict__ x, int64_t ldx, int64_t n, int64_t cols, uint16_t* __restrict__ out) {
  const int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x, per = cols / 8;
  if (id >= n * per) return;
  const int64_t row = id / per, col = id % per * 8;
  const float4 u = *reinterpret_cast<const float4*>(x + row * ldx + col), v = *reinterpret_cast<const float4*>(x + row * ldx + col + 4);
  float r[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
  for (int s = 2; s >= 0; --s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = split_pair(r[2 * i], r[2 * i + 1]);
    *reinterpret_cast<uint4*>(out + (s * n + row) * cols + col) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

struct Plan {
  int mt, tok_tiles, row_tiles, whole, split;
  size_t planes_at, part_at, bytes;
};

Plan make_plan(int x_type, int64_t n, const PackedShape& p) {
  Plan g{};
  const int slots = 2 * device_cu_count();          // two workgroups a compute unit
  g.mt = 4;
  g.tok_tiles = int((n + 32 * g.mt - 1) / (32 * g.mt));
  g.row_tiles = int((p.rows + kTileRows - 1) / kTileRows);
  const int tiles = g.tok_tiles * g.row_tiles;
  g.whole = tiles / slots * slots;
  const int rest = tiles - g.whole;
  const int stages = int(p.kblocks) * (x_type == CAFEQ_F32 ? 3 : 1);
  g.split = rest == 0 ? 1 : std::max(1, std::min(slots / rest, stages / 8));
  if (g.split == 1) g.whole = tiles;
  g.planes_at = 0;
  g.part_at = x_type == CAFEQ_F32 ? align_up(size_t(n) * size_t(p.cols) * 6, 256) : 0;
  g.bytes = g.part_at + size_t(tiles - g.whole) * g.split * 32 * g.mt * kTileRows * sizeof(float);
  return g;
}

template <bool I8, int MT, int FG>
void launch_fg(const GemmArgs& a, bool sx, unsigned nwg, hipStream_t st) {
  constexpr size_t lds = 2 * 32 * MT * Form<I8>::kRowBytes;
  if constexpr (I8) {
    if (sx) {
      hipLaunchKernelGGL((packed_gemm_kernel<I8, MT, FG, true>), dim3(nwg), dim3(kThreads), lds + 2 * (kBlockK / FG) * 32 * MT * 4, st, a);
      return;
    }
  }
  hipLaunchKernelGGL((packed_gemm_kernel<I8, MT, FG, false>), dim3(nwg), dim3(kThreads), lds, st, a);
}

template <bool I8, int MT>
void launch_mt(const GemmArgs& a, int fg, bool sx, unsigned nwg, hipStream_t st) {
  switch (fg) {
    case 128: launch_fg<I8, MT, 128>(a, sx, nwg, st); break;
    case 64: launch_fg<I8, MT, 64>(a, sx, nwg, st); break;
    default: launch_fg<I8, MT, 32>(a, sx, nwg, st); break;
  }
}

}  // namespace

size_t packed_gemm_bytes(int x_type, int64_t n, const PackedShape& p) { return make_plan(x_type, n, p).bytes; }

int launch_packed_gemm(const PackedCall& c, void* ws, hipStream_t st) {
  const Plan g = make_plan(c.x_type, c.n, c.p);
  GemmArgs a{};
  a.packed = c.packed; a.p = c.p; a.n = c.n; a.y = c.y; a.ldy = c.ldy; a.ydtype = c.ydtype;
  a.xscales = c.xscales; a.xgroups = c.xgroups; a.wunits = c.wunits; a.xunits = c.xunits;
  a.planes = 1;
  a.x = static_cast<const uint8_t*>(c.x);
  a.ldx = c.ldx * (c.x_type == CAFEQ_I8 ? 1 : 2);
  if (c.x_type == CAFEQ_F32) {
    uint16_t* planes = reinterpret_cast<uint16_t*>(static_cast<char*>(ws) + g.planes_at);
    const int64_t pieces = c.n * (c.p.cols / 8);
    hipLaunchKernelGGL(split_planes_of_x_kernel, dim3(unsigned((pieces + 255) / 256)), dim3(256), 0, st, static_cast<const float*>(c.x), c.ldx, c.n,
                       c.p.cols, planes);
    CAFEQ_CHECK_LAUNCH();
    a.x = reinterpret_cast<const uint8_t*>(planes);
    a.ldx = c.p.cols * 2;
    a.plane = c.n * c.p.cols * 2;
    a.planes = 3;
  }
  a.tok_tiles = g.tok_tiles; a.row_tiles = g.row_tiles; a.whole = g.whole; a.split = g.split;
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + g.part_at);
  const int rest = g.tok_tiles * g.row_tiles - g.whole;
  const unsigned nwg = unsigned(g.whole + rest * g.split);
  const bool sx = c.x_type == CAFEQ_I8 && c.xgroups > 1;
  if (c.x_type == CAFEQ_I8) launch_mt<true, 4>(a, c.fg, sx, nwg, st);
  else launch_mt<false, 4>(a, c.fg, false, nwg, st);
  CAFEQ_CHECK_LAUNCH();
  if (rest) {
    const bool per_token = c.x_type == CAFEQ_I8 && !sx;
    hipLaunchKernelGGL(packed_join_kernel<4>, dim3(32 * 4 * kTileRows / 256, rest), dim3(256), 0, st, a, per_token);
    CAFEQ_CHECK_LAUNCH();
  }
  return CAFEQ_OK;
}

}  // namespace cafeq
