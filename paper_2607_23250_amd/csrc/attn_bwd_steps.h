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

// The kernels that sum dK and dV hold P and dS in fp16.  That is enough where LSE is that
// of q and k: P is at most 1 and, with max |dO| and max |V| scaled to [1, 2), |dP - D| below
// 2^11.  In a backward from 8-bit checkpoints (LOOSE) LSE is that of q and k before they were
// rounded, and P = exp(S - LSE) has no such bound: scores of some hundreds move by 10 and
// more, and above 65504 the sums turn infinite or NaN and stay so.  Sums that ended so are
// formed once more by wide_step.  (The look at them: causal backward of 4096 tokens, 8 / 2
// heads, d = 64, 124.5 us without and 126.6 with it; of 32768, 32 / 8 heads, 10.2 and 10.1 ms.)
template <int N>
__device__ __forceinline__ bool not_finite(const f32x16 (&x)[N]) {
  bool r = false;
  static_for<N>([&](auto i) {
    static_for<16>([&](auto e) { r |= !(fabsf(x[i][int(e)]) < INFINITY); });
  });
  return r;
}
// dV += dO^T P and dK += Q^T dS over the rows lower <= iq < upper (both less 8 kg) of one
// record at Qs.  S and dP as in the kernels (their operands and offsets: see there); P and dS
// as a bf16 number and a bf16 rest, 16 bits together and the range of fp32; Q^T and dO^T turned to
// bf16, which holds them (they were bf16, scaled by a power of two).
template <int D>
__device__ __forceinline__ void wide_step(const bf16 *Qs, int l, const int (&qoff)[2],
                                          const int (&troff)[2], const f16x8 &ones3,
                                          const f16x8 (&kf)[D / 16], const f16x8 (&vf)[D / 16],
                                          float c2s, int lower, int upper, f32x16 (&dka)[D / 32],
                                          f32x16 (&dva)[D / 32]) {
  constexpr int Q_EL = kRows * D;
  const bf16 *Ag = Qs + 2 * Q_EL + 8 * l;
  const bf16 *rp[2] = {Qs + qoff[0], Qs + qoff[1]};
  const f16 *tp[2] = {reinterpret_cast<const f16 *>(Qs) + troff[0],
                      reinterpret_cast<const f16 *>(Qs) + troff[1]};
  f32x16 sa = mfma32h(*reinterpret_cast<const f16x8 *>(Ag), ones3, mfma_zero_c());
  f32x16 pa = mfma32h(*reinterpret_cast<const f16x8 *>(Ag + kAugEl / 2), ones3, mfma_zero_c());
  static_for<D / 16>([&](auto c) {
    sa = mfma32h(*reinterpret_cast<const f16x8 *>(rp[c & 1] + 1024 * (c >> 1)), kf[c], sa);
    pa = mfma32h(*reinterpret_cast<const f16x8 *>(rp[c & 1] + Q_EL + 1024 * (c >> 1)), vf[c], pa);
  });
  bf16x8 p16[2][2], s16[2][2];   // [rest][16 rows]
  static_for<16>([&](auto r) {
    constexpr int iq = 16 * (r >> 3) + (r & 7);
    const float p = fast_exp2(iq >= lower && iq < upper ? sa[int(r)] * c2s : -INFINITY);
    const float s = p * pa[int(r)];
    p16[0][r >> 3][r & 7] = static_cast<bf16>(p);
    s16[0][r >> 3][r & 7] = static_cast<bf16>(s);
    p16[1][r >> 3][r & 7] = static_cast<bf16>(p - static_cast<float>(p16[0][r >> 3][r & 7]));
    s16[1][r >> 3][r & 7] = static_cast<bf16>(s - static_cast<float>(s16[0][r >> 3][r & 7]));
  });
  auto turned = [&](int at) {
    const f16x8 x = lds_tr16x2h(tp[0] + at, tp[1] + at);
    bf16x8 y;
    static_for<8>([&](auto i) { y[int(i)] = static_cast<bf16>(static_cast<float>(x[int(i)])); });
    return y;
  };
  static_for<D / 32>([&](auto dt) {
    static_for<2>([&](auto c) {
      constexpr int at = 128 * c + 1024 * dt;
      const bf16x8 o = turned(Q_EL + at), q = turned(at);
      static_for<2>([&](auto rest) {
        dva[dt] = mfma32(o, p16[rest][c], dva[dt]);
        dka[dt] = mfma32(q, s16[rest][c], dka[dt]);
      });
    });
  });
}

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
