// Windowed attention (gfx950): preparation passes and the gradients of sink keys over
// far rows.  The forward and dQ kernels are in attn_window_fwd.hip and attn_window_dq.hip;
// the dK / dV kernel is that of the causal calls (attn_bwd.hip), instantiated with WIN.
//
// The row at sample-local position p attends the keys k <= p of its own sample with
// p - k < size or k < sinks.  Work per row is bounded by the window, so key blocks outside
// it are never visited: a forward or dQ item walks the blocks of sinks, then those from the
// first one in the window of its first row to the one of its last row; a dK / dV item (128
// keys) walks the rows from its first key to the window's end of its last key.
//
// Sink keys are attended by all later rows of their sample.  In a long sample these
// far rows are much more than a window, and of the 128 keys of their dK / dV item only the
// few sinks count for them; win_sink_kernel sums them in items of their own, 32 keys wide.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "attn_bwd_steps.h"
#include "attn_common.h"
#include "attn_win_items.h"
#include "errors.h"

namespace libra {

__global__ __launch_bounds__(kPrepThreads) void win_alone_kernel(WinPrep a) {
  __shared__ WinPrepLds lds;
  clear_win_header(a.hdr, a.grid, a.max_items, 0, 0);
  prep_win(a, lds, 0, 1);
}
__global__ __launch_bounds__(kPrepThreads) void win_clear_kernel(int32_t *hdr, int grid,
                                                                 int64_t max_items) {
  clear_win_header(hdr, grid, max_items, 0, 0);
}
__global__ __launch_bounds__(kPrepThreads) void win_items_kernel(WinPrep a) {
  __shared__ WinPrepLds lds;
  prep_win(a, lds, blockIdx.x, gridDim.x);
}

// Workgroups that build the items of a call: one for about 8 rounds of units.
static unsigned prep_blocks(const WinPrep &p) {
  const int64_t units = p.n_q * (int64_t)p.h_q / (kRows * 4);
  const int64_t b = units / (8 * kPrepThreads) + 1;
  return (unsigned)(b < 32 ? 32 : b < 128 ? b : 128);
}

void launch_win_prep_fwd(const WinPrep &p, hipStream_t st) {
  if (p.n_q * (int64_t)p.h_q <= kWinAlonePairs) {
    hipLaunchKernelGGL(win_alone_kernel, dim3(1), dim3(kPrepThreads), 0, st, p);
    return;
  }
  hipLaunchKernelGGL(win_clear_kernel, dim3(1), dim3(kPrepThreads), 0, st, p.hdr, p.grid,
                     p.max_items);
  hipLaunchKernelGGL(win_items_kernel, dim3(prep_blocks(p)), dim3(kPrepThreads), 0, st, p);
}

// ---------------------------------------------------------------------------
// Backward preparation.
__global__ __launch_bounds__(kPrepThreads) void win_bwd_clear_kernel(WinPrep q, WinBwdPrep b,
                                                                     int grid_kv) {
  if (blockIdx.x == 0) {
    clear_win_header(b.hdr, q.grid, q.max_items, grid_kv, b.max_items, b.tops);
    return;
  }
  const int64_t i0 = (int64_t)(blockIdx.x - 1) * kPrepThreads + threadIdx.x;
  const int64_t step = (int64_t)(gridDim.x - 1) * kPrepThreads;
  for (int64_t i = i0; i < b.n; i += step)
    b.samples[i] = WinSample{0, INT32_MAX, INT32_MAX, -1, INT32_MAX, 0, -1, 0, 0};
  for (int64_t i = i0; i < b.n_blocks; i += step) b.blocks[i] = WinBlock{INT32_MAX, -1, 0};
}

// One tile: the samples and key blocks that its rows reach.
__device__ __forceinline__ void win_tile(const WinBwdPrep &a, int64_t t) {
  const libra_tile_t tl = a.tiles[t];
  const int tid = threadIdx.x;
  if (!tile_ok(tl, a.n_q, a.n_kv, a.h_q)) {
    if (tid == 0) atomicAdd(&a.hdr[kBadTiles], 1);
    return;
  }
  bool odd = false;
  const unsigned long long bits =
      group_bits(tl.head_begin, tl.head_end, a.h_q / a.h_kv, odd);
  if (odd && tid == 0) atomicOr(&a.hdr[kOddHeads], 1);
  const int64_t j0 = upper_bound64(a.cu, a.n, tl.q_begin) - 1;
  const int64_t j1 = upper_bound64(a.cu, a.n, tl.q_end - 1);   // one past the last sample
  const int sink_kb = (a.win.sinks + kBwdBK - 1) / kBwdBK;
  // the fragment in sample j, every `step`th key block of it from `first` on
  auto fragment = [&](int64_t j, int first, int step) {
    const int64_t c0 = a.cu[j], c1 = a.cu[j + 1];
    const int la = (int)((tl.q_begin > c0 ? tl.q_begin : c0) - c0);
    const int lb = (int)((tl.q_end < c1 ? tl.q_end : c1) - c0);
    if (la >= lb) return;   // rows past the last sample
    const bool far = far_sample(a.win, a.far_rows, c1 - c0, a.n_kv - c0);
    WinSample &s = a.samples[j];
    if (first == 0) {
      atomicMax(&s.ext, lb);
      atomicMin(&s.beg, la);
      if (far && lb > a.win.size) {
        atomicMin(&s.flo, max(la, a.win.size));
        atomicMax(&s.fhi, lb);
        atomicMin(&s.t0, (int)t);
        atomicMax(&s.t1, (int)t);
        atomicOr(&s.fmask, bits);
      }
    }
    WinBlock *blocks = a.blocks + block_place(c0, j);
    const int kb0 = first_key_block(la, a.win);
    auto reach = [&](int kb, bool walk) {
      if (walk) {
        atomicMin(&blocks[kb].t0, (int)t);
        atomicMax(&blocks[kb].t1, (int)t);
      }
      atomicOr(&blocks[kb].mask, bits);
    };
    for (int kb = kb0 + first; kb <= (lb - 1) / kBwdBK; kb += step) reach(kb, true);
    for (int kb = first; kb < min(sink_kb, kb0); kb += step)
      if (!far || lb > (int64_t)a.win.size + kb * kBwdBK) reach(kb, !far);
  };
  // few samples: all threads share the key blocks of each; else a thread to a sample
  if (j1 - j0 <= 16)
    for (int64_t j = j0; j < j1 && j < a.n; ++j) fragment(j, tid, kPrepThreads);
  else
    for (int64_t j = j0 + tid; j < j1 && j < a.n; j += kPrepThreads) fragment(j, 0, 1);
}
// The dQ items (`item_blocks` workgroups) and the tiles' reach (one workgroup each).
__global__ __launch_bounds__(kPrepThreads) void win_tiles_kernel(WinPrep q, WinBwdPrep b,
                                                                 unsigned item_blocks) {
  __shared__ WinPrepLds lds;
  if (blockIdx.x < item_blocks) prep_win(q, lds, blockIdx.x, item_blocks);
  else win_tile(b, blockIdx.x - item_blocks);
}

// Workgroup 0: the WinSink records and the items of the far rows: parts of equal row ranges,
// at most kSinkParts more of them than records.
__device__ __forceinline__ void win_far_items(const WinBwdPrep &a, int32_t *wsum,
                                              unsigned long long *total_rows) {
  const int tid = threadIdx.x, nsb = sink_blocks(a.win), per = a.h_kv * nsb;
  if (tid == 0) *total_rows = 0;
  __syncthreads();
  int nfar = 0;
  for (int64_t j0 = 0; j0 < a.n; j0 += kPrepThreads) {
    const int64_t j = j0 + tid;
    const bool far = j < a.n && a.samples[j].fhi > 0;
    int all;
    const int at = nfar + block_scan(far, wsum, all);
    if (far) {
      a.samples[j].far = at * per;
      a.far_list[at] = (int32_t)j;
      const WinSample s = a.samples[j];
      atomicAdd(total_rows, (unsigned long long)(s.fhi - s.flo) *
                                (unsigned)(nsb * __builtin_popcountll(s.fmask)));
    }
    nfar += all;
  }
  __threadfence();
  __syncthreads();
  const unsigned long long total = *total_rows;
  // one item for each CU, counting the odd end that every record can have: with twice as
  // many the kernel took 144 us on a 32K pack with a 16K sample, now 117
  const long long want = min(max(a.cus - nfar * per, a.cus / 2), kSinkParts);
  const long long c = (long long)((total + want - 1) / want);
  const long long chunk = c > kSinkPartRows ? (c + kRows - 1) / kRows * kRows : kSinkPartRows;
  int count = 0;
  for (int e0 = 0; e0 < nfar * per; e0 += kPrepThreads) {
    const int e = e0 + tid;
    int np = 0, j = 0, g = 0, sb = 0, r0 = 0;
    WinSample s{};
    if (e < nfar * per) {
      j = a.far_list[e / per];
      g = e % per / nsb;
      sb = e % nsb;
      s = a.samples[j];
      r0 = max(s.flo, a.win.size + 32 * sb);
      if (s.fmask >> g & 1ull && r0 < s.fhi) np = (int)((s.fhi - r0 + chunk - 1) / chunk);
    }
    int all;
    int at = count + block_scan(np, wsum, all);
    count += all;
    if (e < nfar * per) a.sinks[e] = WinSink{at, np};
    for (int p = 0; p < np; ++p, ++at)
      a.sink_items[at] = BwdItem{j, sb, g, at, (int32_t)(r0 + p * chunk),
                                 (int32_t)(p + 1 == np ? s.fhi : r0 + (p + 1) * chunk), s.t0,
                                 s.t1};
  }
  if (tid == 0) {
    a.hdr[kSinkItems] = count;
    a.hdr[kSinkItems + 1] = nfar * per;
  }
}

// The dK / dV items, by KV head, then key block; and (workgroup 0) those of the far rows.
// Calls that cut them (a.parts > 1) have a single workgroup for it, so that slots and split
// records are numbered the same from one call to the next.
__global__ __launch_bounds__(kPrepThreads) void win_kv_items_kernel(WinBwdPrep a) {
  __shared__ int32_t wsum[kPrepThreads / 64];
  __shared__ int32_t base;
  __shared__ unsigned long long total_rows;
  const int tid = threadIdx.x;
  if (blockIdx.x == 0) {
    if (a.win.sinks > 0) win_far_items(a, wsum, &total_rows);
    return;
  }
  const int64_t places = a.n_blocks * a.h_kv;
  int splits = 0;
  const unsigned blocks = gridDim.x - 1, block = blockIdx.x - 1;
  const int64_t share = (places + blocks - 1) / blocks;
  const int64_t pa = share * block, pb = pa + share < places ? pa + share : places;
  for (int64_t p0 = pa; p0 < pb; p0 += kPrepThreads) {
    const int64_t p = p0 + tid;
    BwdItem it{};
    int has = 0, end_row = 0;   // end_row: of the rows that the item can meet
    if (p < pb) {
      const int g = (int)(p / a.n_blocks);
      const int64_t at = p - g * a.n_blocks;
      const WinBlock b = a.blocks[at];
      if (b.mask >> g & 1ull) {
        // the last sample whose block 0 is at or before this place
        int64_t lo = 0, hi = a.n;
        while (hi - lo > 1) {
          const int64_t mid = (lo + hi) >> 1;
          if (block_place(a.cu[mid], mid) <= at) lo = mid; else hi = mid;
        }
        const int64_t c0 = a.cu[lo], len = a.cu[lo + 1] - c0;
        const int kb = (int)(at - block_place(c0, lo));
        // rows up to the window of the last key; inline sinks: all
        const int64_t end = (int64_t)kb * kBwdBK + kBwdBK - 1 + a.win.size;
        const bool all = kb * kBwdBK < a.win.sinks &&
                         !far_sample(a.win, a.far_rows, len, a.n_kv - c0);
        it = BwdItem{(int32_t)lo, kb, g, -1, 0,
                     all || end > INT32_MAX ? INT32_MAX : (int32_t)end, b.t0, b.t1};
        has = 1;
        end_row = min(it.r1, a.samples[lo].ext);
      }
    }
    int all;
    const int at = block_scan(has, wsum, all);
    if (tid == 0) base = all ? atomicAdd(&a.hdr[kBwdQ + kXcds], all * a.parts) : 0;
    __syncthreads();
    const int64_t to = base + (int64_t)at * a.parts;
    if (has && to + a.parts <= a.max_items) {
      if (a.parts > 1) {
        // equal ranges of whole 32-row blocks; the slots of an item are numbered by its place
        const int first = it.kb * kBwdBK, np = a.parts;
        const int per = max(kRows, ((end_row - first + np - 1) / np + kRows - 1) / kRows * kRows);
        const int n = (int)(to / np);
        a.splits[n] = BwdSplit{it, n * np, np, 0, 0};
        const int r1 = it.r1;
        for (int q = 0; q < np; ++q) {
          it.slot = n * np + q;
          it.r0 = q ? first + q * per : 0;
          it.r1 = q + 1 < np ? min(first + (q + 1) * per, r1) : r1;
          a.items[to + q] = it;
        }
      } else {
        a.items[to] = it;
      }
    }
    splits += all;
  }
  if (a.parts > 1 && tid == 0) a.hdr[kBwdSplits] = splits;
}

void launch_win_prep_bwd(const WinPrep &q, const WinBwdPrep &b, int grid_kv, hipStream_t st) {
  const int64_t clear = (b.n + b.n_blocks) / kPrepThreads + 1;
  hipLaunchKernelGGL(win_bwd_clear_kernel, dim3(1 + (unsigned)(clear < 256 ? clear : 256)),
                     dim3(kPrepThreads), 0, st, q, b, grid_kv);
  const unsigned item_blocks = q.n_q * (int64_t)q.h_q <= kWinAlonePairs ? 1 : prep_blocks(q);
  hipLaunchKernelGGL(win_tiles_kernel, dim3(item_blocks + (unsigned)b.T), dim3(kPrepThreads), 0,
                     st, q, b, item_blocks);
  const int64_t places = b.parts > 1 ? 1 : b.n_blocks * b.h_kv / kPrepThreads + 1;
  hipLaunchKernelGGL(win_kv_items_kernel, dim3(1 + (unsigned)(places < 128 ? places : 128)),
                     dim3(kPrepThreads), 0, st, b);
}

// ---------------------------------------------------------------------------
// dK and dV of 32 sink keys of a KV head, over a range of the sample's far rows.  The
// products are those of the dK / dV kernel (queries on M, this lane's key on N); each wave
// holds all 32 keys and takes every fourth step (32 rows x two heads), head by head, through
// two LDS stages of its own, so that no wave waits for another until the four sums are
// added up.  With few sinks one of the 32 columns in eight or so counts, so the products do
// not matter; bound by the latency of the records (a 32K pack with a 16K sample, 32 / 8 heads:
// 250 MB in 117 us, one workgroup to a CU).
// LOOSE: as in the dK / dV kernel.
template <int D, bool LOOSE>
__global__ __launch_bounds__(kThreads, 1) __attribute__((amdgpu_waves_per_eu(1, 1))) void
win_sink_kernel(const f16 *__restrict__ k, const f16 *__restrict__ v,
                const f16 *__restrict__ rec, WinBwdPrep a, float c2,
                float *__restrict__ parts) {
  using S = KvShape<D>;
  constexpr int NC = D / 16, NT = D / 32, LOADS = S::HEAD_EL / 512;   // LOADS: KiB of a record
  static_assert(LOADS <= 63, "vmcnt range");
  extern __shared__ __attribute__((aligned(16))) bf16 smem[];
  const int tid = threadIdx.x, l = tid & 63, ln = l & 31, kg = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h_kv = a.h_kv, G = a.h_q / h_kv;
  const int32_t *hdr = a.hdr;
  const float s_q = fp16_scale((uint32_t)hdr[kMaxAbs + 0], false);
  const float s_k = fp16_scale((uint32_t)hdr[kMaxAbs + 2], false);
  const float c2s = c2 / (s_q * s_k);
  const int prow = perm32(ln);
  const int qoff[2] = {rec_at(prow, kg), rec_at(prow, 2 + kg)};
  int troff[2];
  {
    const int grp = l >> 4, i = (l & 15) >> 2, r = l & 3;
    static_for<2>([&](auto hf) {
      troff[hf] = rec_at(8 * (grp >> 1) + 4 * hf + i, 2 * (grp & 1) + (r & 1)) + 4 * (r >> 1);
    });
  }
  f16x8 ones3;
  static_for<8>([&](auto i) { ones3[int(i)] = f16(kg == 0 && i < 3 ? 1.f : 0.f); });
  bf16 *stage = smem + w * S::STAGE_EL;
  const uint32_t stage_at = lds_addr(stage);
  const int count = hdr[kSinkItems];

  for (int idx = blockIdx.x; idx < count; idx += gridDim.x) {
    const BwdItem item = a.sink_items[idx];
    const int64_t key0 = a.cu[item.sample], len = a.cu[item.sample + 1] - key0;
    const int kl = 32 * item.kb + ln;
    const bool key_ok = kl < a.win.sinks && kl < len;
    f16x8 kf[NC], vf[NC];
    static_for<NC>([&](auto c) {
      static_for<8>([&](auto i) { kf[c][int(i)] = f16(0.f); vf[c][int(i)] = f16(0.f); });
      if (key_ok) {
        const size_t off = ((size_t)(key0 + kl) * h_kv + item.g) * D + 16 * c + 8 * kg;
        kf[c] = *reinterpret_cast<const f16x8 *>(k + off);
        vf[c] = *reinterpret_cast<const f16x8 *>(v + off);
      }
    });
    wait_vm_known();
    f32x16 dva[NT], dka[NT];
    // sums this wave's part; WIDE: whatever the size of P
    auto sum_up = [&](auto wide_t) {
      constexpr bool WIDE = decltype(wide_t)::value;
      static_for<NT>([&](auto dt) {
        dva[dt] = mfma_zero_c();
        dka[dt] = mfma_zero_c();
      });
      StepIter<true> it{a.tiles, (int64_t)item.t1 + 1, a.n_q, a.n_kv, key0, key0 + item.r0,
                  key0 + item.r1, a.h_q, item.g, G, 0, 2 * S::HEAD_EL / 1024};
      it.start(item.t0);
      // this wave's units: the heads of every fourth step, the copy of the next one under way
      // while one is computed
      int n = 0, hb = 0;
      auto skip = [&]() {   // to the next step of this wave
        for (; it.valid && (n & (kWaves - 1)) != w; ++n) it.next();
      };
      struct Unit {
        int lower, upper;   // rows of the block that count for this lane's key, less 8 kg
      };
      auto copy = [&](int buf) {
        const int qb = it.qb(), first = kl + a.win.size - qb;   // first row past the window
        const Unit u{max(it.lo(), min(first, kRows)) - 8 * kg, (key_ok ? it.hi() : 0) - 8 * kg};
        const char *src = reinterpret_cast<const char *>(rec) +
                          (uniform64(it.rec + hb * (S::HEAD_EL / 512)) << 10);
        const uint32_t dst = stage_at + (uint32_t)(buf * S::HEAD_EL * sizeof(bf16));
        static_for<LOADS / 4>([&](auto i) { g2l_run<4>(src + 4096 * i, 16u * l, dst + 4096u * i); });
        if constexpr (LOADS % 4 != 0)
          g2l_run<LOADS % 4>(src + LOADS / 4 * 4096, 16u * l, dst + LOADS / 4 * 4096u);
        if (hb == 0 && it.two()) {
          hb = 1;
        } else {
          hb = 0;
          it.next();
          ++n;
          skip();
        }
        return u;
      };
      skip();
      bool more = it.valid;
      Unit next{};
      if (more) next = copy(0);
      for (int buf = 0; more; buf ^= 1) {
        const Unit u = next;
        more = it.valid;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the other stage's reads are done
        if (more) {
          next = copy(buf ^ 1);
          wait_vm_n<LOADS>();
        } else {
          wait_vm();
        }
        const bf16 *Qs = stage + buf * S::HEAD_EL;
        const bf16 *Ag = Qs + 2 * S::Q_EL + 8 * l;
        const bf16 *rp[2] = {Qs + qoff[0], Qs + qoff[1]};
        const f16 *tp[2] = {reinterpret_cast<const f16 *>(Qs) + troff[0],
                            reinterpret_cast<const f16 *>(Qs) + troff[1]};
        if constexpr (WIDE) {
          wide_step<D>(Qs, l, qoff, troff, ones3, kf, vf, c2s, u.lower, u.upper, dka, dva);
          continue;
        }
        f32x16 sa = mfma32h(*reinterpret_cast<const f16x8 *>(Ag), ones3, mfma_zero_c());
        f32x16 pa =
            mfma32h(*reinterpret_cast<const f16x8 *>(Ag + kAugEl / 2), ones3, mfma_zero_c());
        static_for<NC>([&](auto c) {
          sa = mfma32h(*reinterpret_cast<const f16x8 *>(rp[c & 1] + 1024 * (c >> 1)), kf[c], sa);
          pa = mfma32h(*reinterpret_cast<const f16x8 *>(rp[c & 1] + S::Q_EL + 1024 * (c >> 1)),
                       vf[c], pa);
        });
        f16x8 p16[2], s16[2];
        static_for<16>([&](auto r) {
          constexpr int iq = 16 * (r >> 3) + (r & 7);
          const float x = iq >= u.lower && iq < u.upper ? sa[int(r)] * c2s : -INFINITY;
          const float p = fast_exp2(x);
          p16[r >> 3][r & 7] = static_cast<f16>(p);
          s16[r >> 3][r & 7] = static_cast<f16>(p * pa[int(r)]);
        });
        static_for<NT>([&](auto dt) {
          static_for<2>([&](auto c) {
            constexpr int at = 128 * c + 1024 * dt;
            dva[dt] = mfma32h(lds_tr16x2h(tp[0] + S::Q_EL + at, tp[1] + S::Q_EL + at), p16[c],
                              dva[dt]);
            dka[dt] = mfma32h(lds_tr16x2h(tp[0] + at, tp[1] + at), s16[c], dka[dt]);
          });
        });
      }
    };
    sum_up(std::false_type{});
    if constexpr (LOOSE)
      if (__builtin_amdgcn_ballot_w64(not_finite(dka) || not_finite(dva))) sum_up(std::true_type{});
    // the waves' sums, each in its own stage, then added in wave order
    static_assert(2 * NT * 16 * 64 * sizeof(float) <= S::STAGE_EL * sizeof(bf16), "fits");
    float *ex = reinterpret_cast<float *>(stage);
    static_for<NT>([&](auto dt) {
      static_for<16>([&](auto r) {
        ex[(dt * 16 + r) * 64 + l] = dka[dt][int(r)];
        ex[((NT + dt) * 16 + r) * 64 + l] = dva[dt][int(r)];
      });
    });
    __syncthreads();
    float *out = parts + (size_t)item.slot * sink_part_floats(D);
    for (int x = w; x < 2 * NT; x += kWaves) {
      const int which = x / NT, dt = x % NT;
      for (int r = 0; r < 16; ++r) {
        float s = 0.f;
        for (int u = 0; u < kWaves; ++u)
          s += reinterpret_cast<const float *>(smem + u * S::STAGE_EL)[(x * 16 + r) * 64 + l];
        out[which * 32 * D + ln * D + 32 * dt + 16 * (r >> 3) + 8 * kg + (r & 7)] = s;
      }
    }
    __syncthreads();
  }
}

// Adds up the parts of every WinSink in order, into its first slot.
template <int D>
__global__ __launch_bounds__(256) void win_sink_sum_kernel(const WinSink *__restrict__ sinks,
                                                           const int32_t *__restrict__ hdr,
                                                           float *__restrict__ parts) {
  constexpr int PF = (int)sink_part_floats(D), WG = PF / 4 / 256;   // workgroups of a record
  const int count = hdr[kSinkItems + 1] * WG;
  for (int e = blockIdx.x; e < count; e += gridDim.x) {
    const WinSink s = sinks[e / WG];
    if (s.parts < 2) continue;
    float4 *p = reinterpret_cast<float4 *>(parts + (size_t)s.base * PF) + e % WG * 256 +
                threadIdx.x;
    float4 x = p[0];
#pragma unroll 8
    for (int i = 1; i < s.parts; ++i) {
      const float4 y = p[(size_t)i * (PF / 4)];
      x.x += y.x;
      x.y += y.y;
      x.z += y.z;
      x.w += y.w;
    }
    p[0] = x;
  }
}

template <int D, bool LOOSE>
static int launch_sinks(const f16 *k16, const f16 *v16, const f16 *rec, const WinBwdPrep &b,
                        float c2, float *parts, int cus, hipStream_t st) {
  if (int rc = reserve_lds<&win_sink_kernel<D, LOOSE>>(KvShape<D>::SMEM)) return rc;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(win_sink_kernel<D, LOOSE>), dim3(cus), dim3(kThreads),
                     KvShape<D>::SMEM, st, k16, v16, rec, b, c2, parts);
  hipLaunchKernelGGL(win_sink_sum_kernel<D>, dim3(cus * 2), dim3(256), 0, st, b.sinks, b.hdr,
                     parts);
  return LIBRA_OK;
}
int launch_win_sinks(int d, bool loose, const f16 *k16, const f16 *v16, const f16 *rec,
                     const WinBwdPrep &b, float c2, float *parts, int cus, hipStream_t st) {
  const auto launch = d == 128 ? (loose ? launch_sinks<128, true> : launch_sinks<128, false>)
                               : (loose ? launch_sinks<64, true> : launch_sinks<64, false>);
  return launch(k16, v16, rec, b, c2, parts, cus, st);
}

}  // namespace libra
