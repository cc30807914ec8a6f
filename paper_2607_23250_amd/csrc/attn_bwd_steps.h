// Shared by the dK / dV kernels: the steps that attend a block of keys, and the LDS
// stage that they land in.
#pragma once

#include "attn_common.h"

namespace libra {

__device__ __forceinline__ unsigned long long ld_agent(const unsigned long long *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Bit set of the KV heads whose query groups intersect [hb, he); `odd` is set
// if it covers an odd number of heads of one of them.
__device__ __forceinline__ unsigned long long group_bits(int hb, int he, int G, bool &odd) {
  unsigned long long m = 0;
  for (int g = hb / G; g * G < he; ++g) {
    m |= 1ull << g;
    odd |= ((min(he, (g + 1) * G) - max(hb, g * G)) & 1) != 0;
  }
  return m;
}

template <int D>
struct KvShape {
  static constexpr int Q_EL = kRows * D;
  static constexpr int HEAD_EL = rec_els(D);                  // Q, dO, aug of one head
  static constexpr int STAGE_EL = 2 * HEAD_EL;                // a step is two query heads
  static constexpr int NSTAGE = 4;                            // LDS ring of steps
  static_assert((NSTAGE & (NSTAGE - 1)) == 0, "ring index by mask");
  static constexpr int LOADS = STAGE_EL / 512 / kWaves;       // 1 KiB copies per wave per step
  static_assert(LOADS * 512 * kWaves == STAGE_EL, "every wave copies as much");
  static constexpr size_t SMEM = NSTAGE * STAGE_EL * sizeof(bf16);
  static_assert((NSTAGE - 2) * LOADS <= 63, "vmcnt range");
};

// Walks the steps (32-row query block x two query heads) that attend one KV
// block: tiles in list order, query blocks in row order, heads in order.  Per
// fragment (one tile's rows of the sample) everything a step needs is
// precomputed, so that advancing is a few 32-bit scalar operations plus one
// running 64-bit record offset.
//
// LANES: the lanes of the wave look at 64 tiles at once for the next one with rows of the
// item.  A windowed item meets few of its candidates, and one tile after another cost up
// to 0.5 us each (the far rows of a 16K sample, 16 tiles x 2 head shards: 159 us, 145 with
// this search).
template <bool LANES>
struct StepIter {
  const libra_tile_t *tiles;
  int64_t T, n_q, n_kv, key0, p0, p1;   // rows at positions [p0, p1)
  int h_q, g, G, kloc0, rkib;   // rkib: KiB of a record
  // fragment
  int64_t t;                // tile index
  int nm, lo0, hin, qb0;    // blocks; lo of block 0; hi of the last block; q_loc of its row 0
  int h0, h1;
  // position
  int mi, h;
  int64_t rec;              // offset of the record of (block, h), in KiB
  bool valid;

  // the first tile from `from` on with rows of the item (T: none)
  __device__ int64_t find(int64_t from) const {
    const int lane = threadIdx.x & 63;
    for (; from < T; from += 64) {
      bool has = false;
      if (from + lane < T) {
        const libra_tile_t tl = tiles[from + lane];
        const int64_t pb = tl.q_begin > p0 ? tl.q_begin : p0;
        const int64_t pe = tl.q_end < p1 ? tl.q_end : p1;
        has = tile_ok(tl, n_q, n_kv, h_q) && pb < pe && pe > key0 + kloc0 &&
              tl.head_begin < (g + 1) * G && tl.head_end > g * G;
      }
      const unsigned long long m = __builtin_amdgcn_ballot_w64(has);
      if (m) return from + __builtin_ctzll(m);
    }
    return T;
  }
  __device__ bool seek() {
    if constexpr (LANES) t = find(t);
    for (; t < T; ++t) {
      const libra_tile_t tl = tiles[t];
      if (!tile_ok(tl, n_q, n_kv, h_q)) continue;
      const int64_t pb = tl.q_begin > p0 ? tl.q_begin : p0;
      const int64_t pe = tl.q_end < p1 ? tl.q_end : p1;
      if (pb >= pe) continue;
      h0 = max(tl.head_begin, g * G);
      h1 = min(tl.head_end, (g + 1) * G);
      if (h0 >= h1) continue;
      const int64_t fra = tl.q_row + (pb - tl.q_begin);
      const int64_t frb = fra + (pe - pb);
      const int64_t qla = pb - key0;
      const int64_t first = fra + (kloc0 > qla ? kloc0 - qla : 0);
      if (first >= frb) continue;
      const int64_t mf = first / kRows, ml = (frb - 1) / kRows;
      const int64_t row0 = mf * kRows;
      nm = (int)(ml - mf + 1);
      lo0 = (int)(fra > row0 ? fra - row0 : 0);
      hin = (int)(frb - ml * kRows);
      qb0 = (int)(qla - (fra - row0));
      mi = 0;
      h = h0;
      rec = (mf * h_q + h0) * rkib;
      return true;
    }
    return false;
  }
  __device__ void start(int64_t first) { t = first; valid = seek(); }
  // steps are pairs of query heads (h, h + 1); two() is false for the last
  // step of an odd head count
  __device__ void next() {
    if ((h += 2) < h1) {
      rec += 2 * rkib;
      return;
    }
    rec += (int64_t)((h_q - (h - 2 - h0)) * rkib);   // back by the heads advanced within this block
    h = h0;
    if (++mi < nm) return;
    ++t;
    valid = seek();
  }
  __device__ bool two() const { return h + 1 < h1; }
  __device__ int lo() const { return mi == 0 ? lo0 : 0; }
  __device__ int hi() const { return mi == nm - 1 ? hin : kRows; }
  __device__ int qb() const { return qb0 + kRows * mi; }        // q_loc of the block's row 0
};

}  // namespace libra
