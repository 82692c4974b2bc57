// Products with packed 4-bit weights for many tokens: tiles on the 32x32 matrix instructions.
//   y[t][o] = sum over units of s[o][unit] (sx[t][unit]) sum_{c in unit} q[o][c] x[t][c]
// A workgroup of four or eight waves owns 32 MT tokens; a wave owns all of them and 32 NT rows of the weight.  A stage is 128 columns:
// activations, packed weights and scales go to a ring in LDS asynchronously, up to five stages ahead; a wave unpacks its rows' codes once for all
// the tokens.  Bound by the vector instructions that unpack codes and take a unit's sums up in float32 (conversion, multiply-add), beside the
// matrix instructions: 4608 x 36864, 4096 tokens of 8 bits, a scale each: 684 us, 2.03 POP/s (vector issue 72 % of the cycles, matrix pipe
// 50 %); 14336 x 3584, 512 tokens in bfloat16 59 us, 890 TFLOP/s.  Between those and few tokens by the weights' stream: 36864 x 4608, 32 tokens
// of 8 bits, a scale each 29 us from memory, 3.0 TB/s (25 from the memory-side cache).  Shorter units and grouped scales take their sums up more often:
// 36864 x 4608, 3000 tokens of 8 bits in groups of 128 / 64 / 32 621 / 765 / 1066 us, with a scale per group of the activations too 706 / 980 / 1549.
#include "cafeq_common.hpp"
#include "cafeq_internal.hpp"
#include "packed.hpp"

namespace cafeq {
namespace {

using i32x16 = __attribute__((__vector_size__(16 * sizeof(int)))) int;
using f32x16 = __attribute__((__vector_size__(16 * sizeof(float)))) float;

// waves of a workgroup: eight where a stage of four leaves room for no more than two of its kind on a compute unit
constexpr int tile_waves(bool i8, int mt, int nt) { return mt * nt >= (i8 ? 8 : 4) ? 8 : 4; }

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
  uint32_t winv, xinv;
  int64_t n;
  void* y;
  int64_t ldy;
  int ydtype;
  int tok_tiles, row_tiles;  // tiles of the workgroups
  int whole;              // tiles that one workgroup takes whole; of the others every one goes to `split` of them
  int split;
  float* part;            // [tile - whole][split][tokens x rows of a tile], in the accumulators' order
};

// tile number -> (token tile, row tile): token tiles of a group of eight side by side, so that workgroups that run together share
// activations and weights in their L2
__device__ __forceinline__ void place(int id, const GemmArgs& a, int* tt, int* rt) {
  const int per = 8 * a.row_tiles, g = id / per, in = id % per;
  const int size = min(8, a.tok_tiles - 8 * g);
  *tt = 8 * g + in % size;
  *rt = in / size;
}

// The matrix instructions over a stage's 128 columns, in kParts runs of four; lane l of an operand holds row (or token) l % 32, lane
// half h = l / 32
template <bool I8> struct Form;
template <> struct Form<true> {
  using Frag = i32x4;
  using Acc = i32x16;
  static constexpr int kRowBytes = 128;   // a token's 128 columns
  static constexpr int kParts = 1;        // instruction i: 32 columns, half h their 16 h + 0 .. 15
  // q0, q1: the row's chunks h and h + 2, each with 16 columns of either 64
  static __device__ __forceinline__ Frag unpack(const uint4& q0, const uint4& q1, int, int i) {
    const uint4& q = i & 1 ? q1 : q0;
    const uint32_t d0 = i < 2 ? q.x : q.z, d1 = i < 2 ? q.y : q.w;
    return i32x4{int(low16(d0)), int(high16(d0)), int(low16(d1)), int(high16(d1))};
  }
  static __device__ __forceinline__ int chunk(int, int i, int h) { return 2 * i + h; }
  static __device__ __forceinline__ int swizzle(int row) { return row >> 1 & 7; }   // two rows fill the 64 banks
  static __device__ __forceinline__ Acc mul(const Frag& x, const Frag& b, const Acc& c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(x, b, c, 0, 0, 0); }
};
template <> struct Form<false> {
  using Frag = bf16x8_t;
  using Acc = f32x16;
  static constexpr int kRowBytes = 256;
  static constexpr int kParts = 2;        // instruction i of part p: of the block of 32 2 p + i / 2, half h its 16 h + 8 (i % 2) + 0 .. 7
  static __device__ __forceinline__ Frag unpack(const uint4& q0, const uint4& q1, int p, int i) {
    const uint4& q = i >> 1 ? q1 : q0;
    return bf16_codes(p ? (i & 1 ? q.w : q.z) : (i & 1 ? q.y : q.x));
  }
  static __device__ __forceinline__ int swizzle(int row) { return row & 15; }
  static __device__ __forceinline__ int chunk(int p, int i, int h) { return 4 * (2 * p + (i >> 1)) + 2 * h + (i & 1); }
  static __device__ __forceinline__ Acc mul(const Frag& x, const Frag& b, const Acc& c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, b, c, 0, 0, 0); }
};

// What a workgroup holds in LDS: a ring of stages, as many as leave room for eight waves on the compute unit.  All of a stage --
// activations, weights, scales -- is requested asynchronously, so that a wave knows how many requests follow those of a stage (weights
// loaded to registers instead cost the compiler's waits: 3584 x 14336 and 64 tokens 28 us against 20, 1024 tokens in bfloat16 209 against 143).
template <bool I8, int MT, int NT, int FG, bool SX>
struct Lds {
  static constexpr int kWaves = tile_waves(I8, MT, NT), kThreads = 64 * kWaves;
  static constexpr int kTok = 32 * MT, kUnits = kBlockK / FG;
  static constexpr int kX = kTok * Form<I8>::kRowBytes;              // a stage: activations,
  static constexpr int kW = 32 * NT * kWaves * 64;                   // weights,
  static constexpr int kSw = kWaves * kUnits * 256;                  // their scales [wave][unit][64],
  static constexpr int kSx = SX ? kUnits * kThreads * 4 : 0;         // scales of the activations [unit][threads]
  static constexpr int kStage = kX + kW + kSw + kSx;
  static constexpr int kRoom = 160 * 1024 / (8 / kWaves);            // eight waves a compute unit
  static constexpr int kRing = kRoom / kStage < 2 ? 2 : kRoom / kStage > 6 ? 6 : kRoom / kStage;
  static constexpr int kBytes = kRing * kStage;
  // requests of a wave for a stage
  static constexpr int kDma = kX / 16 / kThreads + kW / 16 / kThreads + kUnits * (SX ? 2 : 1);
};

// 16 (4) bytes a lane from `src` + `off` to LDS address `to` + 16 (4) times the lane, asynchronously.  Opaque to the compiler, which would
// otherwise drain every request before each LDS read; the addresses assume that dynamic LDS starts at 0.
__device__ __forceinline__ void lds_dma16(uint32_t to, uint32_t off, const void* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(src) : "memory");
}
__device__ __forceinline__ void lds_dma4(uint32_t to, uint32_t off, const void* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(off), "s"(src) : "memory");
}

template <bool I8, int MT, int NT, int FG, bool SX>
__global__ __launch_bounds__(64 * tile_waves(I8, MT, NT), 2) void packed_gemm_kernel(const GemmArgs a) {
  using F = Form<I8>;
  using L = Lds<I8, MT, NT, FG, SX>;
  constexpr int kWaves = L::kWaves, kThreads = L::kThreads;
  constexpr int ROWB = F::kRowBytes, CH = ROWB / 16;
  constexpr int NDMA = L::kX / 16 / kThreads;        // requests of a thread and stage
  constexpr int UPB = kBlockK / FG;                 // units of a stage
  constexpr int RUNS = UPB > F::kParts ? UPB / F::kParts : 1, SPU = 4 / RUNS;   // runs of SPU instructions that a part's sums are taken up after
  constexpr int TROWS = 32 * NT * kWaves;
  constexpr int TOK = 32 * MT;
  extern __shared__ __align__(16) unsigned char smem[];
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
  const int64_t row0 = int64_t(rt) * TROWS + wave * 32 * NT; // the wave's first row

  // Requests of the activations: a thread's piece i is 16 bytes of token row i * RSTEP + tid / CH (past the last one: that one's).
  // The chunks of a token lie in LDS at their number XOR the token's swizzle, so that the operand reads of 16 tokens fall on distinct banks.
  constexpr int RSTEP = kThreads / CH;
  const uint32_t ldx = uint32_t(a.ldx), rmax = uint32_t(last) * ldx, rfirst = uint32_t(tid / CH) * ldx;
  const uint32_t ch = uint32_t((tid % CH) ^ F::swizzle(tid / CH)) * 16u;
  const uint32_t tail = uint32_t(a.p.cols - int64_t(nkb - 1) * kBlockK) * (ROWB / kBlockK);   // bytes of a token in the last block
  const uint8_t* xbase = a.x + t0 * a.ldx;
  auto dma = [&](int plane, int kb, int slot) __attribute__((always_inline)) {
    const uint8_t* src = xbase + plane * a.plane + int64_t(kb) * ROWB;
    const uint32_t in = kb == nkb - 1 && ch >= tail ? 0u : ch;
    const uint32_t to = uint32_t(slot * L::kStage) + uint32_t(wave) * 1024u;
#pragma unroll
    for (int i = 0; i < NDMA; ++i) lds_dma16(to + uint32_t(i) * (kThreads * 16u), min(rfirst + uint32_t(i * RSTEP) * ldx, rmax) + in, src);
  };
  // the wave's scales by row; rows past the matrix read its last tile
  const int64_t first = min(row0 / kRowTile, a.p.row_tiles - 1), srow = row0 + min(lane, 32 * NT - 1);
  const uint32_t soff = uint32_t(((min(srow / kRowTile, a.p.row_tiles - 1) - first) * a.p.groups * kRowTile + (srow & 15)) * 4);
  const uint8_t* sbase = a.packed + a.p.scales_at + first * a.p.groups * (kRowTile * 4);
  auto group_w = [&](int kb, int u) { return min(unit_group(kb * UPB + u, a.wunits, a.winv), int(a.p.groups) - 1); };
  auto group_x = [&](int kb, int u) { return min(unit_group(kb * UPB + u, a.xunits, a.xinv), int(a.xgroups) - 1); };
  auto request = [&](int plane, int kb, int slot) __attribute__((always_inline)) {
    dma(plane, kb, slot);
    const uint32_t to = uint32_t(slot * L::kStage + L::kX);
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) {       // the workgroup's tiles of 16 rows kWaves i + wave, as they lie in memory
      const int64_t tile = min(int64_t(rt) * (TROWS / kRowTile) + kWaves * i + wave, a.p.row_tiles - 1);
      lds_dma16(to + uint32_t(kWaves * i + wave) * 1024u, uint32_t(lane) * 16u, a.packed + (tile * nkb + kb) * 1024);
    }
#pragma unroll
    for (int u = 0; u < UPB; ++u) {
      lds_dma4(to + L::kW + uint32_t(wave * UPB + u) * 256u, soff, sbase + group_w(kb, u) * (kRowTile * 4));
      if constexpr (SX)
        lds_dma4(to + L::kW + L::kSw + uint32_t(u * kThreads + wave * 64) * 4u, uint32_t(min(tid, last)) * uint32_t(a.xgroups * 4),
                 a.xscales + t0 * a.xgroups + group_x(kb, u));
    }
  };

  f32x16 y[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) y[m][t][r] = 0.f;

  constexpr int AHEAD = L::kRing - 1;
  int plane = s0 / nkb, kb = s0 % nkb, slot = 0;     // of the stage that is multiplied
  int rplane = plane, rkb = kb, rslot = 0;           // of the one that is requested next (past the last one: the last one again)
  auto request_next = [&]() __attribute__((always_inline)) {
    request(rplane, rkb, rslot);
    rslot = rslot + 1 == L::kRing ? 0 : rslot + 1;
    if (rplane * nkb + rkb + 1 < s1 && ++rkb == nkb) { rkb = 0; ++rplane; }
  };
  for (int i = 0; i < AHEAD; ++i) request_next();
  for (int s = s0; s < s1; ++s) {
    // this stage's requests: all but those of the stages after it
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * L::kDma) : "memory");
    __syncthreads();
    if constexpr (!I8) {
      // past the matrix's columns LDS holds others of the token, of which an infinity times a code of zero would be no number
      if (kb == nkb - 1 && tail < uint32_t(ROWB)) {
        if (ch >= tail)
#pragma unroll
          for (int i = 0; i < NDMA; ++i) *reinterpret_cast<uint4*>(smem + slot * L::kStage + (i * kThreads + tid) * 16) = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
      }
    }
    request_next();
    if (++kb == nkb) { kb = 0; ++plane; }
    const unsigned char* wt = smem + slot * L::kStage + L::kX;
    const float* xs = reinterpret_cast<const float*>(wt + L::kW + L::kSw);
    typename F::Frag b[F::kParts][NT][4];
    float sc[NT][UPB];
    uint4 w[NT][2];                                  // the lane's chunks h and h + 2 of a row
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const unsigned char* at = wt + ((wave * NT + t) * 2 + (l31 >> 4)) * 1024 + (h * 16 + (l31 & 15)) * 16;
      w[t][0] = *reinterpret_cast<const uint4*>(at);
      w[t][1] = *reinterpret_cast<const uint4*>(at + 512);
#pragma unroll
      for (int u = 0; u < UPB; ++u) sc[t][u] = *reinterpret_cast<const float*>(wt + L::kW + (wave * UPB + u) * 256 + (t * 32 + l31) * 4);
    }
    auto unpack = [&](int part, int f) __attribute__((always_inline)) { b[part][f / 4][f % 4] = F::unpack(w[f / 4][0], w[f / 4][1], part, f % 4); };
#pragma unroll
    for (int f = 0; f < 4 * NT; ++f) unpack(0, f);
    const unsigned char* xt = smem + slot * L::kStage + l31 * ROWB;
    const int sz = F::swizzle(l31);
    slot = slot + 1 == L::kRing ? 0 : slot + 1;
    // Tiles one after another, (token tile, run, row tile).  While a tile's instructions run, the one before it is taken up in
    // float32: from the second instruction on, when the last one's result is there.  Where a unit spans both parts of a stage and the
    // registers hold all tiles' accumulators, they are kept from part to part and taken up once; the next part's codes are unpacked meanwhile.
    constexpr int PER = NT * RUNS, TILES = MT * PER;
    constexpr bool KEEP = F::kParts > 1 && UPB == 1;
    constexpr int ACCS = KEEP ? TILES : 2;
    typename F::Acc acc[ACCS];
#pragma unroll
    for (int part = 0; part < F::kParts; ++part) {
      typename F::Frag x[4];
      auto read_x = [&](int m, int i) __attribute__((always_inline)) {
        x[i] = *reinterpret_cast<const typename F::Frag*>(xt + m * 32 * ROWB + (F::chunk(part, i, h) ^ sz) * 16);
      };
      auto take = [&](int j, int q0, int q1) __attribute__((always_inline)) {
        const int m = j / PER, u = UPB > 1 ? part * UPB / F::kParts + j / NT % RUNS : 0, t = j % NT;
#pragma unroll
        for (int v = q0; v < q1; ++v) {
          f32x4 f;
          if constexpr (SX) f = *reinterpret_cast<const f32x4*>(xs + u * kThreads + m * 32 + 8 * v + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = float(acc[j % ACCS][4 * v + e]);
            y[m][t][4 * v + e] = fmaf(SX ? z * f[e] : z, sc[t][u], y[m][t][4 * v + e]);
          }
        }
      };
      const bool taken = !KEEP || part == F::kParts - 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) read_x(0, i);
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
        const int m = j / PER, u = j / NT % RUNS, t = j % NT;
#pragma unroll
        for (int i = 0; i < SPU; ++i) {
          acc[j % ACCS] = F::mul(x[u * SPU + i], b[part][t][u * SPU + i], i == 0 && !(KEEP && part) ? typename F::Acc{} : acc[j % ACCS]);
          if (t == NT - 1 && m + 1 < MT) read_x(m + 1, u * SPU + i);
          __builtin_amdgcn_sched_barrier(0);
          if (part + 1 < F::kParts && (j * SPU + i) % (MT * RUNS * SPU / 4) == 0) unpack(part + 1, (j * SPU + i) / (MT * RUNS * SPU / 4));
          if (j > 0 && taken) {
            if (SPU == 4) take(j - 1, i == 0 ? 0 : i - 1, i == 0 ? 0 : i == 3 ? 4 : i);
            else if (SPU == 2) take(j - 1, i, i == 0 ? 1 : 4);
            else take(j - 1, 0, 4);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (taken) take(TILES - 1, 0, 4);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // requests past the last stage

  if (piece >= 0) {
    float* out = a.part + int64_t(piece) * (TOK * TROWS) + wave * (MT * NT * 16 * 64) + lane;
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
      const float f = (I8 && !SX && tok <= last ? a.xscales[t0 + tok] : 1.f) * code_unit(I8);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int64_t row = row0 + t * 32 + l31;
        if (tok <= last && row < a.p.rows) store_y(a.y, a.ydtype, (t0 + tok) * a.ldy + row, y[m][t][r] * f);
      }
    }
}

// The pieces of a tile in order, to Y: 32 tiles of 128 x 512 in 8 pieces each, 67 MB of partial sums, 19 us (3.5 TB/s).
__global__ __launch_bounds__(256) void packed_join_kernel(const GemmArgs a, int mt, int nt, int waves, bool per_token, float unit) {
  const int size = 32 * mt * 32 * nt * waves;
  const int tile = blockIdx.y, e = blockIdx.x * 256 + threadIdx.x;
  int tt, rt;
  place(a.whole + tile, a, &tt, &rt);
  const int lane = e & 63, r = e >> 6 & 15, at = e >> 10, t = at % nt, m = at / nt % mt, wave = at / nt / mt;   // as the kernel leaves them
  const int64_t tok = int64_t(tt) * 32 * mt + m * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
  const int64_t row = int64_t(rt) * (32 * nt * waves) + (wave * nt + t) * 32 + (lane & 31);
  if (tok >= a.n || row >= a.p.rows) return;
  const float* p = a.part + int64_t(tile) * a.split * size + e;
  float v = 0.f;
  for (int k = 0; k < a.split; ++k) v += p[int64_t(k) * size];
  store_y(a.y, a.ydtype, tok * a.ldy + row, v * ((per_token ? a.xscales[tok] : 1.f) * unit));
}

// float32 activations as three planes of bfloat16, the small parts first: hi + mid + lo exactly (bound by memory, 10 bytes an activation)
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
  int mt, nt, waves, tok_tiles, row_tiles, whole, split;
  size_t part_at, bytes;
};

// What a stage of a tile takes, in us: on a compute unit alone, and with a second workgroup there (units of 128 and one scale a token, whose costs stand
// for those of shorter units and grouped scales too; 4608 columns, one or two
// workgroups a compute unit and, of the larger tiles, thousands).
struct TileCost { int mt, nt; float alone, paired; };
constexpr TileCost kTilesI8[] = {{1, 1, 0.48f, 0.69f}, {2, 1, 0.64f, 0.92f}, {2, 2, 1.1f, 1.75f}, {4, 2, 1.8f, 2.9f}};
constexpr TileCost kTilesBf16[] = {{1, 1, 0.62f, 0.88f}, {2, 1, 0.83f, 1.27f}, {2, 2, 1.38f, 2.2f}};   // 4 x 2 leaves no room for a second workgroup: 5.0

// The tile and the split with the least estimated time.  Tiles that fill rounds of workgroups run whole; of the rest every one is split along
// the columns, as far as that fills the compute units and its partial sums (written, read, a launch more) cost less than it gains.
// 3584 x 14336, 32 tokens of 8 bits, split 1 / 4 / 9 / 18: 60 / 21 / 16 / 18 us; 36864 x 4608 1 / 2 / 4: 26 / 33 / 34.
Plan make_plan(int x_type, int64_t n, const PackedShape& p) {
  Plan best{};
  double least = 1e30;
  const int cus = device_cu_count();
  const int stages = int(p.kblocks) * (x_type == CAFEQ_F32 ? 3 : 1);
  auto consider = [&](const TileCost& c) {
    const int waves = tile_waves(x_type == CAFEQ_I8, c.mt, c.nt), trows = 32 * c.nt * waves, slots = 8 / waves * cus;
    const int64_t tok_tiles = (n + 32 * c.mt - 1) / (32 * c.mt), row_tiles = (p.rows + trows - 1) / trows, tiles = tok_tiles * row_tiles;
    const int64_t whole = tiles / slots * slots, rest = tiles - whole;
    // pieces of so many stages, eight waves a compute unit at a time; 1.5 us to begin and end one
    auto run = [&](int64_t pieces, int64_t depth) {
      const int64_t left = pieces % slots;
      return double(pieces / slots) * (double(depth) * c.paired + 1.5) + (left ? double(depth) * (left > cus || waves == 8 ? c.paired : c.alone) + 1.5 : 0.0);
    };
    for (int64_t split = 1; split == 1 || (split <= stages / 2 && rest * split <= 4 * slots); ++split) {
      const double per = run(whole, stages) + run(rest * split, (stages + split - 1) / split);
      const double join = split == 1 ? 0.0 : 4.0 + double(rest * split) * (32 * c.mt * trows * 4) * 2 / 4.5e6;
      const double t = per + join;
      if (t < least) {
        least = t;
        best.mt = c.mt; best.nt = c.nt; best.waves = waves; best.tok_tiles = int(tok_tiles); best.row_tiles = int(row_tiles);
        best.split = int(split); best.whole = int(split == 1 ? tiles : whole);
        best.bytes = split == 1 ? 0 : size_t(rest * split) * (32 * c.mt * trows * 4);
      }
      if (rest == 0) break;
    }
  };
  if (x_type == CAFEQ_I8) for (const TileCost& c : kTilesI8) consider(c);
  else for (const TileCost& c : kTilesBf16) consider(c);
  best.part_at = x_type == CAFEQ_F32 ? align_up(size_t(n) * size_t(p.cols) * 6, 256) : 0;
  best.bytes += best.part_at;
  return best;
}

template <bool I8, int MT, int NT, int FG, bool SX>
int launch_one(const GemmArgs& a, unsigned nwg, hipStream_t st) {
  constexpr int lds = Lds<I8, MT, NT, FG, SX>::kBytes;
  auto* kern = packed_gemm_kernel<I8, MT, NT, FG, SX>;
  if constexpr (lds > 64 * 1024) {
    static const bool ok = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
    if (!ok) return CAFEQ_ERR_LAUNCH;
  }
  hipLaunchKernelGGL(kern, dim3(nwg), dim3(Lds<I8, MT, NT, FG, SX>::kThreads), lds, st, a);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

template <bool I8, int MT, int NT>
int launch_tile(const GemmArgs& a, int fg, bool sx, unsigned nwg, hipStream_t st) {
  if constexpr (I8) {
    if (sx) return fg == 128 ? launch_one<I8, MT, NT, 128, true>(a, nwg, st) : fg == 64 ? launch_one<I8, MT, NT, 64, true>(a, nwg, st)
                                                                                        : launch_one<I8, MT, NT, 32, true>(a, nwg, st);
  }
  return fg == 128 ? launch_one<I8, MT, NT, 128, false>(a, nwg, st) : fg == 64 ? launch_one<I8, MT, NT, 64, false>(a, nwg, st)
                                                                               : launch_one<I8, MT, NT, 32, false>(a, nwg, st);
}

}  // namespace

size_t packed_gemm_bytes(int x_type, int64_t n, const PackedShape& p) { return make_plan(x_type, n, p).bytes; }

int launch_packed_gemm(const PackedCall& c, void* ws, hipStream_t st) {
  const Plan g = make_plan(c.x_type, c.n, c.p);
  GemmArgs a{};
  a.packed = c.packed; a.p = c.p; a.n = c.n; a.y = c.y; a.ldy = c.ldy; a.ydtype = c.ydtype;
  a.xscales = c.xscales; a.xgroups = c.xgroups; a.wunits = c.wunits; a.xunits = c.xunits; a.winv = c.winv; a.xinv = c.xinv;
  a.planes = 1;
  a.x = static_cast<const uint8_t*>(c.x);
  a.ldx = c.ldx * (c.x_type == CAFEQ_I8 ? 1 : 2);
  if (c.x_type == CAFEQ_F32) {
    uint16_t* planes = static_cast<uint16_t*>(ws);
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
  const bool i8 = c.x_type == CAFEQ_I8, sx = i8 && c.xgroups > 1;
  int rc = CAFEQ_ERR_UNSUPPORTED;
  switch (g.mt * 10 + g.nt) {
    case 11: rc = i8 ? launch_tile<true, 1, 1>(a, c.fg, sx, nwg, st) : launch_tile<false, 1, 1>(a, c.fg, false, nwg, st); break;
    case 21: rc = i8 ? launch_tile<true, 2, 1>(a, c.fg, sx, nwg, st) : launch_tile<false, 2, 1>(a, c.fg, false, nwg, st); break;
    case 22: rc = i8 ? launch_tile<true, 2, 2>(a, c.fg, sx, nwg, st) : launch_tile<false, 2, 2>(a, c.fg, false, nwg, st); break;
    case 42: rc = launch_tile<true, 4, 2>(a, c.fg, sx, nwg, st); break;
  }
  if (rc) return rc;
  if (rest) {
    const int size = 32 * g.mt * 32 * g.nt * g.waves;
    hipLaunchKernelGGL(packed_join_kernel, dim3(size / 256, rest), dim3(256), 0, st, a, g.mt, g.nt, g.waves, i8 && !sx, code_unit(i8));
    CAFEQ_CHECK_LAUNCH();
  }
  return CAFEQ_OK;
}

}  // namespace cafeq
