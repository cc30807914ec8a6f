// Work items of windowed attention, built on the device.
//
// A window bounds an item's key blocks, so items cost about the same and need no
// sorting: they go into one list, in the order (tile, head chunk, 32-row window), so
// that neighbours read the same K / V rows.  Without the sort a call of many rows can
// have many workgroups build its list.
#pragma once

#include "attn_common.h"

namespace libra {

struct WinPrep {
  const int64_t *cu;
  int64_t n;
  const libra_tile_t *tiles;
  int64_t T;
  int h_q, h_kv;
  int64_t n_q, n_kv;
  Window win;
  int32_t *hdr;
  FwdItem *items;
  int64_t max_items;
  int count_bad;
  int grid;        // workgroups that run the items
  int split_grid;  // workgroups that the split rule counts
  int max_parts, idle_only;
  FwdSplit *splits;
};
constexpr int kWinMinSteps = 4;   // a part of a split item walks at least 4 key blocks
// Calls of at most this many (row, query head) pairs have one workgroup build their
// items; it clears the header itself and can split items.
constexpr int64_t kWinAlonePairs = 131072;

struct WinPrepLds {
  int64_t pre[kPrepThreads];   // units before each tile of the batch
  int32_t cu[kCuLds];
  int32_t wsum[3][kPrepThreads / 64];
  long long wunits[kPrepThreads / 64];
  unsigned long long est, items, work, parts;
  int32_t base, nslot, nsplit, bad;
};

// Sums of v over the threads before this one; `total`: over all.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int32_t *wsum, int &total) {
  const int tid = threadIdx.x;
  int inc = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(inc, o);
    if ((tid & 63) >= o) inc += x;
  }
  if ((tid & 63) == 63) wsum[tid >> 6] = inc;
  __syncthreads();
  int before = 0, sum = 0;
  for (int i = 0; i < kPrepThreads / 64; ++i) {
    if (i < (tid >> 6)) before += wsum[i];
    sum += wsum[i];
  }
  total = sum;
  __syncthreads();
  return before + inc - v;
}

// Head chunks (up to 4 query heads of one KV group) of heads [hb, he).
__device__ __forceinline__ int head_chunks(int hb, int he, int G) {
  const int g0 = hb / G, g1 = (he - 1) / G;
  if (g0 == g1) return (he - hb + 3) / 4;
  return ((g0 + 1) * G - hb + 3) / 4 + (g1 - g0 - 1) * ((G + 3) / 4) + (he - g1 * G + 3) / 4;
}
// Chunk c of them: its KV head, first query head and heads.
__device__ __forceinline__ void head_chunk(int hb, int he, int G, int c, int &g, int &h0,
                                           int &nh) {
  g = hb / G;
  int first = hb, end = min(he, (g + 1) * G);
  const int c0 = (end - hb + 3) / 4;
  if (c >= c0) {
    const int cg = (G + 3) / 4;
    g += 1 + (c - c0) / cg;
    c = (c - c0) % cg;
    first = g * G;
    end = min(he, first + G);
  }
  h0 = first + 4 * c;
  nh = min(4, end - h0);
}

// The items of one head chunk whose first row lies in rows [wa, wb) of a tile
// (at most 32 rows): f(item), with its steps in kb1 and, in the place of the sample's index,
// its first key.
template <typename F>
__device__ __forceinline__ void for_each_win_item(const libra_tile_t &t, int64_t wa, int64_t wb,
                                                  const CuView &cu, int64_t n, int g, int h0,
                                                  int nh, const Window &win, F &&f) {
  const int rows_per = kRows * (4 / nh);
  int64_t j = upper_bound64(cu, n, wa) - 1;
  for (; j < n && cu[j] < wb; ++j) {
    const int64_t c0 = cu[j], c1 = cu[j + 1];
    const int64_t pb = t.q_begin > c0 ? t.q_begin : c0;
    const int64_t pe = t.q_end < c1 ? t.q_end : c1;
    const int64_t lim = wb < pe ? wb : pe;
    int64_t k = wa > pb ? (wa - pb + rows_per - 1) / rows_per : 0;
    for (; pb + k * rows_per < lim; ++k) {
      const int64_t rb = k * rows_per;
      const int nrows = (int)(pe - pb - rb < rows_per ? pe - pb - rb : rows_per);
      const int32_t qmin = (int32_t)(pb + rb - c0), qmax = qmin + nrows - 1;
      const int w0 = max(0, qmin - win.size + 1) / kFwdBN;   // first block of the window
      const int far = min((win.sinks + kFwdBN - 1) / kFwdBN, w0);
      f(FwdItem{(int32_t)(t.q_row + (pb + rb - t.q_begin)), qmin, (int32_t)c0, h0, nh, nrows, g, 0,
                far + qmax / kFwdBN + 1 - w0, -1, far, w0 - far});
    }
  }
}

// Clears the header of a windowed call (one workgroup of kPrepThreads): the lists are
// empty, hold up to max_q and max_kv items and are run by grid_q and grid_kv workgroups.
__device__ __forceinline__ void clear_win_header(int32_t *hdr, int grid_q, int64_t max_q,
                                                 int grid_kv, int64_t max_kv) {
  static_assert(kHdrSlots <= kPrepThreads, "a thread to a slot");
  const int tid = threadIdx.x;
  if (tid < kHdrSlots) {
    int v = 0;
    for (int x = 0; x < kXcds; ++x) {
      if (tid == head_slot(kFwdQ, x)) v = (grid_q - x + kXcds - 1) / kXcds;
      if (tid == head_slot(kBwdQ, x)) v = (grid_kv - x + kXcds - 1) / kXcds;
    }
    if (tid == kFwdQ + 2 * kXcds) v = (int)(max_q < INT32_MAX ? max_q : INT32_MAX);
    if (tid == kBwdQ + 2 * kXcds) v = (int)(max_kv < INT32_MAX ? max_kv : INT32_MAX);
    __hip_atomic_store(&hdr[tid], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// One workgroup (gridDim.x = 1, or workgroup 0 when the tiles turn out to cover few
// rows) or many, each with an equal run of the units (tile, head chunk, 32-row window).
//
// Split K: a call with fewer items than twice `split_grid` (with `idle_only`, only if
// whole rounds of them would leave more than a tenth of the workgroups idle) cuts items
// of at least two parts into key ranges of about a quarter of a workgroup's share, as
// the causal calls do; one workgroup then builds the list, and the parts' slots go by
// its order, so that nothing depends on which part runs where.
__device__ __forceinline__ void prep_win(const WinPrep &a, WinPrepLds &lds, unsigned block,
                                         unsigned blocks) {
  const int tid = threadIdx.x, G = a.h_q / a.h_kv;
  const int64_t n = a.n, T = a.T;
  const CuView cu = cu_view(a.cu, n, lds.cu);
  if (tid == 0) {
    lds.est = lds.items = lds.work = lds.parts = 0;
    lds.base = lds.nslot = lds.nsplit = lds.bad = 0;
  }
  __syncthreads();
  // items at least, and the tiles outside the buffers
  {
    unsigned long long est = 0;
    int bad = 0;
    for (int64_t t = tid; t < T; t += kPrepThreads) {
      const libra_tile_t tl = a.tiles[t];
      if (!tile_ok(tl, a.n_q, a.n_kv, a.h_q)) {
        ++bad;
        continue;
      }
      est += (unsigned long long)((tl.q_end - tl.q_begin + 127) / 128) *
             (unsigned)head_chunks(tl.head_begin, tl.head_end, G);
    }
    if (est) atomicAdd(&lds.est, est);
    if (bad) atomicAdd(&lds.bad, bad);
    __syncthreads();
  }
  const bool few = lds.est < 2ull * (unsigned)a.split_grid;
  const bool alone = blocks == 1 || few;
  if (alone && block) return;
  if (tid == 0 && block == 0 && a.count_bad && lds.bad) atomicAdd(&a.hdr[kBadTiles], lds.bad);
  const unsigned nb = alone ? 1 : blocks;

  // every unit of this workgroup: f(tile, first row, end, KV head, first head, heads), by
  // rounds of one unit to a thread (valid says whether it has one), for all threads alike
  auto units = [&](auto &&f) {
    for (int64_t tb = 0; tb < T; tb += kPrepThreads) {
      long long u = 0;
      if (tb + tid < T) {
        const libra_tile_t tl = a.tiles[tb + tid];
        if (tile_ok(tl, a.n_q, a.n_kv, a.h_q))
          u = (tl.q_end - tl.q_begin + kRows - 1) / kRows *
              head_chunks(tl.head_begin, tl.head_end, G);
      }
      long long inc = u;
      for (int o = 1; o < 64; o <<= 1) {
        const long long x = __shfl_up(inc, o);
        if ((tid & 63) >= o) inc += x;
      }
      __syncthreads();   // the batch before is done with `pre`
      if ((tid & 63) == 63) lds.wunits[tid >> 6] = inc;
      __syncthreads();
      long long before = 0, total = 0;
      for (int i = 0; i < kPrepThreads / 64; ++i) {
        if (i < (tid >> 6)) before += lds.wunits[i];
        total += lds.wunits[i];
      }
      lds.pre[tid] = before + inc - u;
      __syncthreads();
      const long long ua = total / nb * block + total % nb * block / nb;
      const long long ub = total / nb * (block + 1) + total % nb * (block + 1) / nb;
      for (long long v0 = ua; v0 < ub; v0 += kPrepThreads) {
        const long long v = v0 + tid;
        const bool valid = v < ub;
        libra_tile_t tl{};
        int64_t wa = 0, wb = 0;
        int g = 0, h0 = 0, nh = 1;
        if (valid) {
          // the last tile with no more units before it
          int lo = 0, hi = kPrepThreads;
          while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (lds.pre[mid] <= v) lo = mid; else hi = mid;
          }
          tl = a.tiles[tb + lo];
          const int64_t windows = (tl.q_end - tl.q_begin + kRows - 1) / kRows;
          const long long r = v - lds.pre[lo];
          const int c = (int)(r / windows);
          wa = tl.q_begin + kRows * (r - c * windows);
          wb = wa + kRows < tl.q_end ? wa + kRows : tl.q_end;
          head_chunk(tl.head_begin, tl.head_end, G, c, g, h0, nh);
        }
        f(valid, tl, wa, wb, g, h0, nh);
      }
    }
  };

  int chunk = 0;   // steps of a part; 0: no item is split
  if (alone && few && a.max_parts > 0) {
    units([&](bool valid, const libra_tile_t &tl, int64_t wa, int64_t wb, int g, int h0, int nh) {
      if (!valid) return;
      unsigned long long items = 0, work = 0;
      for_each_win_item(tl, wa, wb, cu, n, g, h0, nh, a.win, [&](const FwdItem &it) {
        ++items;
        work += (unsigned)it.kb1;
      });
      if (items) {
        atomicAdd(&lds.items, items);
        atomicAdd(&lds.work, work);
      }
    });
    __syncthreads();
    const unsigned long long items = lds.items, work = lds.work, gr = (unsigned)a.split_grid;
    const bool idle = items * 10 < (items + gr - 1) / gr * gr * 9;
    if (items > 0 && items < 2 * gr && (idle || !a.idle_only)) {
      // items longer than C number at most work / C, their parts at most twice that
      const unsigned long long c = (work + 4 * gr - 1) / (4 * gr);
      const unsigned long long fit = (2 * work + a.max_parts - 1) / (unsigned)a.max_parts;
      const unsigned long long m = c > fit ? c : fit;
      chunk = (int)(m > kWinMinSteps ? m : kWinMinSteps);
    }
  }
  // parts of an item (1: whole)
  auto parts_of = [&](const FwdItem &it) {
    return chunk && it.kb1 >= 2 * chunk ? (it.kb1 + chunk - 1) / chunk : 1;
  };
  units([&](bool valid, const libra_tile_t &tl, int64_t wa, int64_t wb, int g, int h0, int nh) {
    int items = 0, slots = 0, cut = 0;
    if (valid)
      for_each_win_item(tl, wa, wb, cu, n, g, h0, nh, a.win, [&](const FwdItem &it) {
        const int np = parts_of(it);
        items += np;
        slots += np > 1 ? np : 0;
        cut += np > 1;
      });
    int all, all_slots = 0, all_cut = 0;
    const int before_items = block_scan(items, lds.wsum[0], all);
    int slot = 0, sp = 0;
    if (chunk) {
      slot = lds.nslot + block_scan(slots, lds.wsum[1], all_slots);
      sp = lds.nsplit + block_scan(cut, lds.wsum[2], all_cut);
    }
    __syncthreads();
    if (tid == 0) {
      if (alone) {
        lds.parts = (unsigned long long)lds.base;
        lds.base += all;
      } else {
        lds.parts = (unsigned)atomicAdd(&a.hdr[kFwdQ + kXcds], all);
      }
      // the run that reaches past the list (overlapping tiles can fill it)
      if ((long long)lds.parts <= a.max_items && (long long)lds.parts + all > a.max_items)
        atomicAdd(&a.hdr[a.count_bad ? kBadTiles : kDqFull], 1);
      lds.nslot += all_slots;
      lds.nsplit += all_cut;
    }
    __syncthreads();
    int64_t at = before_items + (int64_t)lds.parts;
    if (valid)
      for_each_win_item(tl, wa, wb, cu, n, g, h0, nh, a.win, [&](const FwdItem &it) {
        const int np = parts_of(it), per = (it.kb1 + np - 1) / np;
        if (np > 1) a.splits[sp++] = FwdSplit{it, slot, np, 0, 0};
        for (int p = 0; p < np; ++p) {
          FwdItem ip = it;
          if (np > 1) {
            ip.kb0 = p * per;   // < kb1: per <= chunk and (np - 1) chunk < kb1
            ip.kb1 = min((p + 1) * per, it.kb1);
            ip.slot = slot++;
          }
          if (at < a.max_items) a.items[at] = ip;
          ++at;
        }
      });
  });
  if (alone) {
    __syncthreads();
    if (tid == 0) {
      a.hdr[kFwdQ + kXcds] = lds.base;
      a.hdr[kFwdSplits] = lds.nsplit;
      a.hdr[kFwdSplits + 1] = lds.nslot;
    }
  }
}

// ---------------------------------------------------------------------------
// Backward: what the covered rows reach.

// Of a sample: covered rows are among [beg, ext); those past the window of its first key,
// if it is a far sample, among [flo, fhi) of the tiles [t0, t1], in the KV heads of fmask.
struct WinSample {
  int32_t ext, beg;
  int32_t t0, t1, flo, fhi;
  int32_t far;   // a far sample's first WinSink record, or -1
  int32_t pad;
  unsigned long long fmask;
};
// Of a 128-key block: the KV heads in which covered rows attend it, and the tiles that
// its dK / dV items walk.
struct WinBlock {
  int32_t t0, t1;
  unsigned long long mask;
};
// 32 sink keys of a far sample and KV head: their partial sums over far rows are in slots
// [base, base + parts), each sink_part_floats: dK, then dV, 32 keys x D, fp32.
struct WinSink {
  int32_t base, parts;
};
constexpr int kMaxSinks = 1024;
constexpr int kSinkParts = 1024;   // slots beyond one for each WinSink
__host__ __device__ constexpr int sink_blocks(const Window &w) { return (w.sinks + 31) / 32; }
__host__ __device__ constexpr size_t sink_part_floats(int d) { return (size_t)2 * 32 * d; }
// First 128-key block in the window of the row at sample-local position p.
__device__ __forceinline__ int first_key_block(int p, const Window &w) {
  return max(0, p - w.size + 1) / kBwdBK;
}
// Place of a sample's key block 0 among all (a sample's blocks follow one another).
__device__ __forceinline__ int64_t block_place(int64_t first_key, int64_t j) {
  return first_key / kBwdBK + j;
}

struct WinBwdPrep {
  const int64_t *cu;
  int64_t n;
  const libra_tile_t *tiles;
  int64_t T;
  int h_q, h_kv;
  int64_t n_q, n_kv;
  Window win;
  int32_t *hdr;
  WinSample *samples;
  WinBlock *blocks;
  int64_t n_blocks;
  BwdItem *items;
  int64_t max_items;
  WinSink *sinks;       // one for each far sample, KV head and 32 sinks
  int32_t *far_list;    // far samples with covered far rows
  BwdItem *sink_items;  // (sample, 32 sinks, KV head) x far rows
};

// Can a call split an item?  One of two parts or more: its rows' window, the rows (at
// most 128) and the sinks have to reach over that many blocks.
inline bool win_may_split(const Window &w, int64_t n_kv) {
  const int64_t reach = (int64_t)w.size + kFwdPartRows + kFwdBN;
  return (reach < n_kv ? reach : n_kv) / kFwdBN + 1 + (w.sinks + kFwdBN - 1) / kFwdBN >=
         2 * kWinMinSteps;
}

// Arguments of the windowed dQ kernel (attn_window_dq.hip).  q and o, or q8 and o8.
struct WinDq {
  const bf16 *q, *o, *dout, *k, *v;
  Held q8, o8;
  const float *lse;
  const FwdItem *items;
  int32_t *hdr;
  int h_q, h_kv;
  int64_t n_q, nq_pad;
  float scale, c2, d_fix;   // d_fix: see attn_bwd_dq.hip
  Window win;
  bf16 *dq;
  f16 *rec;
  float *stats, *parts;
};
constexpr int kWinDqPerCu = 2;   // workgroups per CU
int launch_win_dq(int d, const WinDq &a, int cus, hipStream_t st);

// Launchers (attn_window.hip).
void launch_win_prep_fwd(const WinPrep &p, hipStream_t st);
// The preparation of a windowed backward: the dQ items (q) and the dK / dV items (b).
void launch_win_prep_bwd(const WinPrep &q, const WinBwdPrep &b, int grid_kv, hipStream_t st);
// The far rows of sink keys: partial sums of dK and dV, one slot a WinSink after it.
int launch_win_sinks(int d, const f16 *k16, const f16 *v16, const f16 *rec, const WinBwdPrep &b,
                     float c2, float *parts, int cus, hipStream_t st);

}  // namespace libra
