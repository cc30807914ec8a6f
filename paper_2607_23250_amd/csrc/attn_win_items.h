// Work items of windowed attention, built on the device.
//
// A window bounds an item's key blocks, so items cost about the same and need no
// sorting: they go into one list, in the order (tile, head chunk, 32-row window), so
// that neighbours read the same K / V rows.  Without the sort a call of many rows can
// have many workgroups build its list.
#pragma once

#include "attn_common.h"

namespace libra {

// A record that no store of the kernel changes, at an address that is the same in every lane:
// a scalar load.  (As a vector load its wait would also be one for the copies under way.)
template <typename T>
__device__ __forceinline__ T load_uniform(const T *p) {
  static_assert(sizeof(T) % 8 == 0, "whole 8 bytes");
  struct Words {
    uint64_t w[sizeof(T) / 8];
  } x;
  const auto *c = (const __attribute__((address_space(4))) uint64_t *)(uintptr_t)p;
  static_for<sizeof(T) / 8>([&](auto i) { x.w[int(i)] = c[int(i)]; });
  return __builtin_bit_cast(T, x);
}

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
  int max_parts;   // 0: no item is split
  FwdSplit *splits;
};
// A part of a split item walks at least 6 key blocks (backward of 4096 tokens, 2 / 1 heads,
// window 4096: 142 us with 4, 132 with 6, 134 with 8; forward of 2000: 34, 38, 42).
constexpr int kWinMinSteps = 6;
// Items of fewer steps than these are not split: the parts' merge takes longer than it saves
// (forward of 4096 tokens, 8 / 2 heads, d = 64, window 1024, 21 steps: 46 us split, 36 whole;
// of 2000 tokens, 2 / 1 heads, 34 steps: 38 split, 43 whole).
constexpr int kWinSplitSteps = 24;
// Calls of at most this many (row, query head) pairs have one workgroup build their
// items; it clears the header itself (16K tokens, window 128 to 256: 8 heads 38 us with one
// workgroup and 39 with many, 32 heads 157 and 140).
constexpr int64_t kWinAlonePairs = 131072;

struct WinTile {   // of a tile, what its items need
  int64_t q_begin, q_end, q_row;
  int32_t head_begin, head_end;
};
struct WinPrepLds {
  WinTile tiles[kPrepThreads];   // a batch of tiles, those outside the buffers without rows
  int64_t pre[kPrepThreads];     // units before each of them
  int32_t cu[kCuLds];
  int32_t wsum[3][kPrepThreads / 64];
  int64_t wunits[kPrepThreads / 64];
  unsigned long long est, items, work;
  int32_t base, at, nslot, nsplit, bad;
};

__device__ __forceinline__ long long wave_sum(long long v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Sums of v over the threads before this one; `total`: over all.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int32_t *wsum, int &total) {
  constexpr int W = kPrepThreads / 64;
  const int tid = threadIdx.x, l = tid & 63;
  int inc = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(inc, o);
    if (l >= o) inc += x;
  }
  if (l == 63) wsum[tid >> 6] = inc;
  __syncthreads();
  int sum = wsum[l & (W - 1)];   // every wave adds up the waves' sums
  for (int o = 1; o < W; o <<= 1) {
    const int x = __shfl_up(sum, o);
    if ((l & (W - 1)) >= o) sum += x;
  }
  total = __shfl(sum, W - 1);
  const int before = __shfl(sum, max((tid >> 6) - 1, 0));
  __syncthreads();
  return (tid >= 64 ? before : 0) + inc - v;
}

// Head chunks (up to 4 query heads of one KV group) of heads [hb, he).
__device__ __forceinline__ int head_chunks(int hb, int he, int G) {
  const int g0 = hb / G, g1 = (he - 1) / G;
  if (g0 == g1) return (he - hb + 3) / 4;
  return ((g0 + 1) * G - hb + 3) / 4 + (g1 - g0 - 1) * ((G + 3) / 4) + (he - g1 * G + 3) / 4;
}
// log2 of the rows of an item of nh heads: 32 (4 / nh).
__device__ __forceinline__ int item_rows_log2(int nh) { return nh == 1 ? 7 : nh == 2 ? 6 : 5; }

// Items of heads [hb, he) x rows that lie in one sample.
__device__ __forceinline__ int64_t items_of(int64_t rows, int hb, int he, int G) {
  auto of = [&](int heads) {
    const int rest = heads & 3, sh = item_rows_log2(rest);
    return heads / 4 * ((rows + kRows - 1) / kRows) +
           (rest ? (rows + (1 << sh) - 1) >> sh : (int64_t)0);
  };
  const int g0 = hb / G, g1 = (he - 1) / G;
  if (g0 == g1) return of(he - hb);
  return of((g0 + 1) * G - hb) + (g1 - g0 - 1) * of(G) + of(he - g1 * G);
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

// The item of one head chunk that starts rb rows into the fragment of tile rows [pb, pe) of
// the sample with first key c0: its steps in kb1 and, in the place of the sample's index, c0.
__device__ __forceinline__ FwdItem win_item(const WinTile &t, int64_t c0, int64_t pb, int64_t pe,
                                            int64_t rb, int rows_per, int g, int h0, int nh,
                                            const Window &win) {
  const int nrows = (int)(pe - pb - rb < rows_per ? pe - pb - rb : rows_per);
  const int32_t qmin = (int32_t)(pb + rb - c0), qmax = qmin + nrows - 1;
  const int w0 = max(0, qmin - win.size + 1) / kFwdBN;   // first block of the window
  const int far = min((win.sinks + kFwdBN - 1) / kFwdBN, w0);
  return FwdItem{(int32_t)(t.q_row + (pb + rb - t.q_begin)), qmin, (int32_t)c0, h0, nh, nrows, g,
                 0, far + qmax / kFwdBN + 1 - w0, -1, far, w0 - far};
}

// The items of one head chunk whose first row lies in rows [wa, wb) of a tile (at most 32
// rows, so at most one of a sample): f(item).
template <typename F>
__device__ __forceinline__ void for_each_win_item(const WinTile &t, int64_t wa,
                                                  int64_t wb, const CuView &cu, int64_t n, int g,
                                                  int h0, int nh, const Window &win, F &&f) {
  const int sh = item_rows_log2(nh);
  int64_t j = upper_bound64(cu, n, wa) - 1;
  for (; j < n && cu[j] < wb; ++j) {
    const int64_t c0 = cu[j], c1 = cu[j + 1];
    const int64_t pb = t.q_begin > c0 ? t.q_begin : c0;
    const int64_t pe = t.q_end < c1 ? t.q_end : c1;
    const int64_t rb = wa > pb ? (wa - pb + (1 << sh) - 1) >> sh << sh : 0;
    if (pb + rb < (wb < pe ? wb : pe)) f(win_item(t, c0, pb, pe, rb, 1 << sh, g, h0, nh, win));
  }
}

// ---------------------------------------------------------------------------
// Calls of single tokens (no more Q rows than tiles) and small ones: no list.  Unit (tile, head
// chunk, part) finds its work itself, which saves the preparation's launch and most of its time
// (64 sequences, 32 / 8 heads: 20 of 239 us; one: 11 of 25).  Unit p of a tile of one row has
// key range p of up to `cuts` of equal length of its item; of a tile with more rows it has every
// parts-th 32-row window from window p on, and whole items.
struct WinRows {
  const int64_t *cu;
  int64_t n;
  const libra_tile_t *tiles;
  int64_t T;
  int h_q, h_kv;
  int64_t n_q, n_kv;
  Window win;
  int32_t *hdr;
  int chunks;   // head chunks of all heads
  int parts;    // units of a tile and chunk
  int cuts;     // key ranges of a single row's item at most
  int64_t units() const { return T * chunks * parts; }
};
// A key range of a single row walks at least 2 key blocks (one sequence, 17 blocks: 13.1 us,
// 14.6 with at least 4), and an item has at most 64 of them (20000 keys, one chunk of 4 heads:
// 22.7 us with up to 32, 18.9 with 64, 19.4 with 256).
constexpr int kRowMinSteps = 2;
constexpr int kRowMaxCuts = 64;
// Key ranges of a single row's item of this many steps.
__device__ __forceinline__ int row_parts(int steps, int cuts) {
  return max(1, min(cuts, steps / kRowMinSteps));
}
// Last sample that begins at or before x (uniform in the wave): guess, then 64-ary search.
__device__ __forceinline__ int64_t sample_at(const int64_t *cu, int64_t n, int64_t x,
                                             int64_t guess) {
  if (guess < n && load_uniform(cu + guess) <= x && x < load_uniform(cu + guess + 1))
    return guess;
  const int lane = threadIdx.x & 63;
  int64_t lo = 0, count = n;   // the answer is among [lo, lo + count)
  while (count > 1) {
    const int64_t step = (count + 63) / 64;
    const int64_t at = lo + lane * step;
    const bool le = lane * step < count && cu[at] <= x;
    const int last = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(le) | 1ull);
    lo += last * step;
    count = count - last * step < step ? count - last * step : step;
  }
  return lo;
}
// Walks the items of one unit; all values are uniform in the workgroup.
struct RowUnit {
  WinTile t;
  int g, h0, nh, p;
  int64_t job;      // (tile, chunk), numbered
  int64_t guess;
  int64_t w, j;     // next window; next sample in it (-1: not looked up)
  bool valid;

  __device__ __forceinline__ RowUnit(const WinRows &a, int64_t unit) {
    job = unit / a.parts;
    p = (int)(unit - job * a.parts);
    guess = job / a.chunks;
    const int c = (int)(job - guess * a.chunks);
    const libra_tile_t tl = load_uniform(a.tiles + guess);
    t = WinTile{tl.q_begin, tl.q_end, tl.q_row, tl.head_begin, tl.head_end};
    valid = tile_ok(tl, a.n_q, a.n_kv, a.h_q);
    if (!valid) return;
    const int G = a.h_q / a.h_kv;
    valid = c < head_chunks(t.head_begin, t.head_end, G);
    if (!valid) return;
    head_chunk(t.head_begin, t.head_end, G, c, g, h0, nh);
    w = one_row() ? 0 : p;
    j = -1;
  }
  __device__ __forceinline__ bool one_row() const { return t.q_end - t.q_begin == 1; }
  // The next item, or false.
  __device__ __forceinline__ bool next(const WinRows &a, FwdItem &it) {
    if (!valid) return false;
    const int sh = item_rows_log2(nh);
    for (;; w += a.parts, j = -1) {
      const int64_t wa = t.q_begin + kRows * w;
      if (wa >= t.q_end) return false;
      const int64_t wb = wa + kRows < t.q_end ? wa + kRows : t.q_end;
      if (j < 0) j = sample_at(a.cu, a.n, wa, guess);
      while (j < a.n) {
        const int64_t c0 = load_uniform(a.cu + j), c1 = load_uniform(a.cu + j + 1);
        if (c0 >= wb) break;
        ++j;
        const int64_t pb = t.q_begin > c0 ? t.q_begin : c0;
        const int64_t pe = t.q_end < c1 ? t.q_end : c1;
        const int64_t rb = wa > pb ? (wa - pb + (1 << sh) - 1) >> sh << sh : 0;
        if (pb + rb >= (wb < pe ? wb : pe)) continue;
        it = win_item(t, c0, pb, pe, rb, 1 << sh, g, h0, nh, a.win);
        if (!one_row()) return true;
        const int np = row_parts(it.kb1, a.cuts), per = (it.kb1 + np - 1) / np;
        valid = false;   // the only one
        if (p * per >= it.kb1) return false;   // per <= kb1: parts past the cuts have none
        if (np > 1) {
          it.kb0 = p * per;
          it.kb1 = min((p + 1) * per, it.kb1);
          it.slot = (int32_t)(job * a.cuts + p);
        }
        return true;
      }
    }
  }
};

// Clears the header of a windowed call (one workgroup of kPrepThreads): the lists are
// empty, hold up to max_q and max_kv items and are run by grid_q and grid_kv workgroups.
__device__ __forceinline__ void clear_win_header(int32_t *hdr, int grid_q, int64_t max_q,
                                                 int grid_kv, int64_t max_kv,
                                                 const ScoreTops &tops = {0, 0}) {
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
    if (tid == kMaxAbs) v = tops.q;
    if (tid == kMaxAbs + 2) v = tops.k;
    __hip_atomic_store(&hdr[tid], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// One workgroup (gridDim.x = 1, or workgroup 0 when the tiles turn out to cover few
// rows) or many, each with an equal run of the units (tile, head chunk, 32-row window).
//
// Split K: a call with fewer items than twice `split_grid` cuts items of at least two parts
// into key ranges of about half a workgroup's share (forward of 12000 tokens, 4 / 2 heads, no
// key outside the window: 268 us with a whole share, 178 with half, 182 with a quarter); one
// workgroup then builds the list, and the parts' slots go by its order, so that nothing
// depends on which part runs where.
__device__ __forceinline__ void prep_win(const WinPrep &a, WinPrepLds &lds, unsigned block,
                                         unsigned blocks) {
  const int tid = threadIdx.x, l = tid & 63, G = a.h_q / a.h_kv;
  const int64_t n = a.n, T = a.T;
  const CuView cu = cu_view(a.cu, n, lds.cu);
  if (tid == 0) {
    lds.est = lds.items = lds.work = 0;
    lds.base = lds.nslot = lds.nsplit = lds.bad = 0;
  }
  __syncthreads();
  // The tiles [tb, tb + kPrepThreads) and the units before each; returns the units of all.
  // `first`: also counts the items at least, and the tiles outside the buffers.
  auto load = [&](int64_t tb, bool first) {
    WinTile wt{};
    int64_t u = 0;
    long long est = 0;
    bool bad = false;
    if (tb + tid < T) {
      const libra_tile_t tl = a.tiles[tb + tid];
      bad = !tile_ok(tl, a.n_q, a.n_kv, a.h_q);
      if (!bad) {
        wt = WinTile{tl.q_begin, tl.q_end, tl.q_row, tl.head_begin, tl.head_end};
        const int chunks = head_chunks(tl.head_begin, tl.head_end, G);
        u = (tl.q_end - tl.q_begin + kRows - 1) / kRows * chunks;
        est = items_of(tl.q_end - tl.q_begin, tl.head_begin, tl.head_end, G);
      }
    }
    if (first) {
      est = wave_sum(est);
      const int b = __builtin_popcountll(__builtin_amdgcn_ballot_w64(bad));
      if (l == 0 && est) atomicAdd(&lds.est, (unsigned long long)est);
      if (l == 0 && b) atomicAdd(&lds.bad, b);
    }
    lds.tiles[tid] = wt;
    long long inc = u;
    for (int o = 1; o < 64; o <<= 1) {
      const long long x = __shfl_up(inc, o);
      if (l >= o) inc += x;
    }
    if (l == 63) lds.wunits[tid >> 6] = inc;
    __syncthreads();
    constexpr int W = kPrepThreads / 64;
    long long sum = lds.wunits[l & (W - 1)];
    for (int o = 1; o < W; o <<= 1) {
      const long long x = __shfl_up(sum, o);
      if ((l & (W - 1)) >= o) sum += x;
    }
    const int64_t total = __shfl(sum, W - 1);
    const long long before = __shfl(sum, max((tid >> 6) - 1, 0));
    lds.pre[tid] = (tid >= 64 ? before : 0) + inc - u;
    __syncthreads();
    return total;
  };
  int64_t total = 0;
  for (int64_t tb = 0; tb < T; tb += kPrepThreads) total = load(tb, true);
  // the header's clearing stores, if this workgroup made them, come before what follows
  wait_vm_known();
  __syncthreads();
  const bool one_batch = T <= kPrepThreads;   // then it stays loaded
  const bool few = lds.est < 2ull * (unsigned)a.split_grid;
  const bool alone = blocks == 1 || few;
  if (alone && block) return;
  if (tid == 0 && block == 0 && a.count_bad && lds.bad) atomicAdd(&a.hdr[kBadTiles], lds.bad);
  const unsigned nb = alone ? 1 : blocks;

  // every unit of this workgroup: f(valid, tile, first row, end, KV head, first head, heads),
  // by rounds of one unit to a thread (valid: it has one), for all threads alike
  auto units = [&](auto &&f) {
    for (int64_t tb = 0; tb < T; tb += kPrepThreads) {
      if (!one_batch) {
        __syncthreads();   // the batch before is done with
        total = load(tb, false);
      }
      const int64_t ua = total / nb * block + total % nb * block / nb;
      const int64_t ub = total / nb * (block + 1) + total % nb * (block + 1) / nb;
      for (int64_t v0 = ua; v0 < ub; v0 += kPrepThreads) {
        const int64_t v = v0 + tid;
        const bool valid = v < ub;
        WinTile tl{};
        int64_t wa = 0, wb = 0;
        int g = 0, h0 = 0, nh = 1;
        if (valid) {
          // the last tile with no more units before it
          int lo = 0, hi = (int)(T - tb < kPrepThreads ? T - tb : kPrepThreads);
          while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (lds.pre[mid] <= v) lo = mid; else hi = mid;
          }
          tl = lds.tiles[lo];
          const int64_t windows = (tl.q_end - tl.q_begin + kRows - 1) / kRows;
          const int64_t r = v - lds.pre[lo];
          const int64_t c = (r | windows) >> 32 ? r / windows
                                                : (int64_t)((uint32_t)r / (uint32_t)windows);
          wa = tl.q_begin + kRows * (r - c * windows);
          wb = wa + kRows < tl.q_end ? wa + kRows : tl.q_end;
          head_chunk(tl.head_begin, tl.head_end, G, (int)c, g, h0, nh);
        }
        f(valid, tl, wa, wb, g, h0, nh);
      }
    }
  };

  int chunk = 0;   // steps of a part; 0: no item is split
  if (alone && few && a.max_parts > 0) {
    units([&](bool valid, const WinTile &tl, int64_t wa, int64_t wb, int g, int h0, int nh) {
      long long items = 0, work = 0;
      if (valid)
        for_each_win_item(tl, wa, wb, cu, n, g, h0, nh, a.win, [&](const FwdItem &it) {
          ++items;
          work += it.kb1;
        });
      items = wave_sum(items);
      work = wave_sum(work);
      if (l == 0 && items) {
        atomicAdd(&lds.items, (unsigned long long)items);
        atomicAdd(&lds.work, (unsigned long long)work);
      }
    });
    __syncthreads();
    const unsigned long long items = lds.items, work = lds.work, gr = (unsigned)a.split_grid;
    if (items > 0 && items < 2 * gr) {
      // items longer than C number at most work / C, their parts at most twice that
      const unsigned long long c = (work + 2 * gr - 1) / (2 * gr);
      const unsigned long long fit = (2 * work + a.max_parts - 1) / (unsigned)a.max_parts;
      const unsigned long long m = c > fit ? c : fit;
      chunk = (int)(m > kWinMinSteps ? m : kWinMinSteps);
    }
  }
  // parts of an item (1: whole)
  auto parts_of = [&](const FwdItem &it) {
    return chunk && it.kb1 >= 2 * chunk ? (it.kb1 + chunk - 1) / chunk : 1;
  };
  units([&](bool valid, const WinTile &tl, int64_t wa, int64_t wb, int g, int h0, int nh) {
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
      __syncthreads();
    }
    if (tid == 0) {
      lds.at = alone ? lds.base : atomicAdd(&a.hdr[kFwdQ + kXcds], all);
      lds.base += all;
      // the run that reaches past the list (overlapping tiles can fill it)
      if (lds.at <= a.max_items && (int64_t)lds.at + all > a.max_items)
        atomicAdd(&a.hdr[a.count_bad ? kBadTiles : kDqFull], 1);
      lds.nslot += all_slots;
      lds.nsplit += all_cut;
    }
    __syncthreads();
    int64_t at = (int64_t)lds.at + before_items;
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
// Rows of a part of far rows at least (backward with 4 sinks: 8192 tokens, 32 / 4 heads, window
// 512: 500 us with 512, 465 with 128 and with 32; 2000 tokens, 8 / 2 heads, window 256: 119 with
// 128, 114 with 32).
constexpr int kSinkPartRows = 32;
constexpr int kSinkParts = 256;      // slots beyond one for each WinSink
__host__ __device__ constexpr int sink_blocks(const Window &w) { return (w.sinks + 31) / 32; }
__host__ __device__ constexpr size_t sink_part_floats(int d) { return (size_t)2 * 32 * d; }
// A sample whose rows reach this far past the window of its first key has the
// gradients of its sink keys summed over those far rows by a kernel of their
// own; in shorter ones the far rows are part of the sink keys' dK / dV items.
// (Backward of 4096 tokens, 8 / 2 heads, window 256, 4 sinks: 196 us with 512, 157 with 256 and
// 128; of 8192, 32 / 4 heads, window 512: 794 with 2048, 474, 449, 446.)
constexpr int kFarRows = 256;
// Is a sample a far one?  `keys`: those from its first to the end of K, which the last may pass;
// the workspace has room for the far samples that fit K side by side.
__device__ __forceinline__ bool far_sample(const Window &w, int far_rows, int64_t len,
                                           int64_t keys) {
  return w.sinks > 0 && (len < keys ? len : keys) > (int64_t)w.size + far_rows;
}
// The far samples of a call number at most min(n, n_kv / (size + far_rows + 1)), each with a
// record and a slot of 64 d floats for 32 sinks of a KV head.  Many of them with many sinks would
// take more than all else in the workspace (400 samples in 262144 keys, 8 KV heads, 1024 sinks, d =
// 128: 3.4 GB), so there the line between far samples and others rises until the slots take no
// more bytes than the fp16 copies of K and V (or 4096 slots, if those are more).  It rises only
// where far samples and sinks are many: then most keys of the samples that it leaves out are sinks,
// and an item of 128 keys is the better form for them (that call, 16 query heads, window 128: 9.6
// ms with 256 rows for all, 5.6 so; 60 samples of 2000, window 8, 1024 sinks: 7.1 and 4.0).
inline int64_t win_far_max(const Window &w, int far_rows, int64_t n, int64_t n_kv) {
  const int64_t fit = n_kv / ((int64_t)w.size + far_rows + 1);
  return w.sinks ? (n < fit ? n : fit) : 0;
}
inline int win_far_rows(const Window &w, int64_t n, int64_t n_kv, int h_kv) {
  const int64_t copies = n_kv * h_kv / 64, room = copies > 4096 ? copies : 4096;
  const int64_t most = w.sinks ? room / ((int64_t)h_kv * sink_blocks(w)) : 0;   // 2 or more
  // n_kv / (size + far_rows + 1) <= most
  return win_far_max(w, kFarRows, n, n_kv) <= most ? kFarRows
                                                   : (int)(n_kv / (most + 1) - w.size);
}
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
  int cus;
  BwdSplit *splits;     // dK / dV items cut into `parts` row ranges each (1: none)
  int parts;
  ScoreTops tops;
  int far_rows;         // see far_sample
};
// Row ranges of a dK / dV item.  A call of few key blocks and KV heads (4K tokens and 2 KV
// heads: 66 items for 256 CUs) cuts each into as many as the CUs hold, of at least 2 row blocks
// (backward of 1000 tokens, 4 / 1 heads, window 300: 106 us with at least 8, 81 with 4, 77 with
// 2), and up to 8 (4096 tokens, 2 / 1 heads, window 4096: 145 us; 163 with up to 4; no less
// with 16).
constexpr int kWinKvMinBlocks = 2;
inline int win_kv_parts(const Window &w, int64_t key_blocks, int h_kv, int cus) {
  const int64_t fit = cus / (key_blocks * h_kv);
  const int64_t most = ((int64_t)w.size + kBwdBK) / (kWinKvMinBlocks * kRows);
  const int64_t n = fit < most ? fit : most;
  return (int)(n < 1 ? 1 : n > 8 ? 8 : n);
}
constexpr int kWinMaxSplits = 512;   // split dK / dV items of a call (more than CUs / 2)

// Steps of an item of up to `rows` rows at most: their window, the rows and the sinks.
inline int64_t win_max_steps(const Window &w, int64_t n_kv, int rows = kFwdPartRows) {
  const int64_t reach = (int64_t)w.size + rows + kFwdBN;
  return (reach < n_kv ? reach : n_kv) / kFwdBN + 1 + (w.sinks + kFwdBN - 1) / kFwdBN;
}
// Can a call split an item?  Shorter ones take less time than their parts' merge.
inline bool win_may_split(const Window &w, int64_t n_kv) {
  return win_max_steps(w, n_kv) >= kWinSplitSteps;
}
// Single tokens beyond this many (tile, head chunk) pairs go through the list.
constexpr int64_t kMaxRowJobs = 1 << 20;
// Other calls without a list have at most this many units (8 / 2 heads, d = 64, window 128:
// 4096 tokens in tiles of 512, 2048 units: 19.9 us, 22.9 with a list; 16384 tokens in tiles of
// 2048, 8192 units, most of them past their tile's end: 55, 39 with a list).
constexpr int64_t kMaxSmallUnits = 4096;

// Arguments of the windowed dQ kernel (attn_window_dq.hip).  q and o, or q8 and o8.
struct WinDq {
  const bf16 *q, *o, *dout;
  const f16 *k16, *v16;
  Held q8, o8;
  const float *lse;
  const FwdItem *items;
  int32_t *hdr;
  int h_q, h_kv;
  int64_t n_q, nq_pad;
  float scale, c2;
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
// The far rows of sink keys: partial sums of dK and dV, one slot a WinSink after it.  `loose`:
// see attn_bwd_steps.h.
int launch_win_sinks(int d, bool loose, const f16 *k16, const f16 *v16, const f16 *rec,
                     const WinBwdPrep &b, float c2, float *parts, int cus, hipStream_t st);

}  // namespace libra
