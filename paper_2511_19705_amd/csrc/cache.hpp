// The cache of keys and values in 8 bits: what its kernels share.
#pragma once
#include "cafeq_common.hpp"
#include "heads.hpp"

namespace cafeq {

constexpr int kCacheDMax = 256;
constexpr int64_t kMaxSeqs = 65535, kMaxHeads = 4096, kMaxKeys = int64_t(1) << 30;

inline int check_cache(const cafeq_cache* c) {
  if (!c || !c->k || !c->v || !c->kscale || !c->vscale || (c->sequences && (!c->table || !c->lengths))) return CAFEQ_ERR_INVALID_ARG;
  if (c->sequences < 0 || c->width < 1 || c->heads < 1 || c->pages < 1 || c->d < 16 || c->d % 16) return CAFEQ_ERR_BAD_SHAPE;
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return CAFEQ_ERR_UNSUPPORTED;
  if (c->d > kCacheDMax || c->heads > kMaxHeads || c->sequences > kMaxSeqs || c->pages > INT32_MAX || c->pages * c->heads > INT32_MAX ||
      int64_t(c->width) * c->block > kMaxKeys)
    return CAFEQ_ERR_UNSUPPORTED;
  if (!aligned_to(c->k, 16) || !aligned_to(c->v, 16) || !aligned_to(c->kscale, 4) || !aligned_to(c->vscale, 4) || !aligned_to(c->table, 4) ||
      !aligned_to(c->lengths, 4) || !aligned_to(c->refs, 4) || !aligned_to(c->missing, 4))
    return CAFEQ_ERR_BAD_ALIGN;
  return CAFEQ_OK;
}

// Rows lo .. hi - 1 of sequence i, within 0 .. n whatever starts holds
struct RowRange { int lo, hi; };
__device__ __forceinline__ RowRange rows_of(const int32_t* starts, int i, int n) {
  RowRange r;
  r.lo = min(max(starts[i], 0), n);
  r.hi = min(max(starts[i + 1], r.lo), n);
  return r;
}
__device__ __forceinline__ int tokens_of(const cafeq_cache& c, int i) { return min(max(c.lengths[i], 0), c.width * c.block); }
// Whether the last reserve found no room: lengths do not count the new tokens then.  (Read without a branch: `any` is readable in any case)
__device__ __forceinline__ bool no_room(const cafeq_cache& c, const int32_t* any) {
  const int lack = *(c.missing ? c.missing : any);
  return c.missing && lack != 0;
}
// page of a block of sequence i, or -1
__device__ __forceinline__ int page_of(const cafeq_cache& c, int i, int block) {
  const int p = c.table[int64_t(i) * c.width + block];
  return p >= 0 && p < c.pages ? p : -1;
}

// Work that goes over all sequences is numbered so that sequence i begins at unit base(i) = floor(starts[i] * mul / div) + extra i; `extra`
// makes room for the units that rows of a sequence touch beyond their number over div / mul.  The sequence of unit w: the last one that
// begins at w or before.  All lanes of a wave look together, 64 sequences a step.
struct Units {
  int mul, div, extra;
  __host__ __device__ int64_t base(int64_t start, int64_t i) const { return start * mul / div + extra * i; }
  int64_t count(int64_t n, int64_t sequences) const { return base(n, sequences); }
};
__device__ __forceinline__ int sequence_of(const Units& u, const int32_t* starts, int sequences, int n, int64_t w) {
  const int lane = threadIdx.x & 63;
  int first = 0, left = sequences;
  while (left > 0) {
    const int step = (left + 63) / 64;
    const int i = first + lane * step;
    const bool in = lane * step < left && u.base(min(max(starts[i], 0), n), i) <= w;
    const int seen = __popcll(__ballot(in));
    if (seen == 0) return -1;
    first += (seen - 1) * step;
    left = step > 1 ? min(step, sequences - first) : 0;
  }
  // (starts out of order may have led elsewhere)
  return sequences > 0 && u.base(min(max(starts[first], 0), n), first) <= w ? first : -1;
}

}  // namespace cafeq
