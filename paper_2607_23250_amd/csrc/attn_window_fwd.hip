// Forward kernel of windowed attention (gfx950).
//
// The mathematics and the work items are the causal forward's (attn_fwd.hip): S^T = K Q^T
// (lane = query), the online softmax, O^T += V^T P^T; up to 4 query heads of one KV group x 32
// rows, a wave each, K and V blocks of 64 keys double-buffered in LDS, two workgroups per CU
// (three at d = 64).  What the window adds:
//   * the item walks steps (step_block): the blocks of sinks, then those of the window;
//   * each wave passes over the 32-key halves of a block in which none of its rows attends a
//     key: with a window of 1024 an item's 18.5 blocks come down to 17.3 (16.1 would have no
//     masked key at all);
//   * a half that some row does not attend whole is masked by element, and a row may have no
//     key in it, so the running max starts at the lowest finite value;
//   * keys that no row of the item attends are not read: in a cache they may hold anything.
// P is rounded to bf16 for its product with V, whose type it shares; the running max, the
// row sum and O stay in fp32, and the sum takes P before the rounding.
// Bound by the matrix cores' share of the cycles and the clock under them (a 32K pack, 32
// heads, window 1024: 603 us, 819 TFLOP/s, busy 42% at 1.86 GHz; the 256K share, window 4096:
// 1787 to 1850 us, 1.03 PFLOP/s, 53% at 1.64); single tokens (WinRows) by reading K and V
// (64 sequences of 6000 keys, 8 KV heads, window 4096: 181 us, 5.5 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "attn_common.h"
#include "attn_win_items.h"
#include "errors.h"

namespace libra {

template <int D>
struct WinFwdShape {
  static constexpr int KC = D / 8;            // 16-byte columns of a K / V row
  static constexpr int K_EL = kFwdBN * D;
  static constexpr int STAGE = 2 * K_EL;      // K and V rows of one key block
  static constexpr int NK = kFwdBN * KC / 64 / kWaves;   // wave loads of 1 KB per tile
  static constexpr size_t SMEM = 2 * STAGE * sizeof(bf16);
  static_assert(NK == 2 || NK == 4, "d = 64 or 128");
};
// Workgroups per CU: at d = 64 the registers of three fit, as in the causal forward (not
// those of the single-token form, which would spill).
template <int D, bool ROWS>
constexpr int kWinFwdPerCu = D == 64 && !ROWS ? 3 : 2;

struct WinFwd {
  const bf16 *q, *k, *v;
  const FwdItem *items;
  int32_t *hdr;
  int h_q, h_kv;
  int64_t n_q;
  float c2;
  bf16 *o;
  float *lse, *parts;
  Window win;
};

// The tiles outside the buffers, counted by one workgroup into the header (`count`: shared).
__device__ __forceinline__ void count_bad_tiles(const WinRows &a, int32_t &count) {
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  int bad = 0;
  for (int64_t t = threadIdx.x; t < a.T; t += kThreads)
    bad += !tile_ok(a.tiles[t], a.n_q, a.n_kv, a.h_q);
  if (bad) atomicAdd(&count, bad);
  __syncthreads();
  if (threadIdx.x == 0) a.hdr[kBadTiles] = count;
}
struct NoRows {};
struct NoUnit {
  __device__ __forceinline__ NoUnit(const NoRows &, int64_t) {}
};

// R: NoRows (the items of the list) or WinRows (no list: the workgroup's items are those of
// one unit; the last workgroup counts the tiles outside the buffers instead).
template <int D, typename R>
__global__ __launch_bounds__(kThreads, (kWinFwdPerCu<D, std::is_same_v<R, WinRows>>)) void
win_fwd_kernel(WinFwd a, R rows) {
  using S = WinFwdShape<D>;
  constexpr bool ROWS = std::is_same_v<R, WinRows>;
  constexpr int NC = D / 16, NT = D / 32;
  extern __shared__ __attribute__((aligned(16))) bf16 smem[];
  __shared__ int32_t s_item[2];
  if constexpr (ROWS) {
    if (blockIdx.x == gridDim.x - 1) {
      count_bad_tiles(rows, s_item[0]);
      return;
    }
  }
  const int tid = threadIdx.x, l = tid & 63, ln = l & 31, kg = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);   // wave index (uniform)
  const int h_q = a.h_q, h_kv = a.h_kv;
  const Window win = a.win;
  // operand reads and staging as in the causal forward; half h of a block is 32 h D elements
  // further
  constexpr int STEP4 = S::KC == 16 ? 128 : 256;   // elements from chunk j to chunk j + 4
  const int prow = perm32(ln);
  const int koff[2] = {swu<S::KC>(prow, kg), swu<S::KC>(prow, 2 + kg)};
  int troff[2];
  {
    const int grp = l >> 4, i = (l & 15) >> 2, r = l & 3;
    static_for<2>([&](auto hf) {
      troff[hf] = swu<S::KC>(8 * (grp >> 1) + 4 * hf + i, 2 * (grp & 1) + (r & 1)) + 4 * (r >> 1);
    });
  }
  uint32_t k_lane[S::NK];
  static_for<S::NK>([&](auto u) {
    const int wl = w + kWaves * u;
    k_lane[u] = 2u * (uint32_t)(swu_row<S::KC>(wl, l) * h_kv * D + 8 * swu_col<S::KC>(wl, l));
  });

  // The items of a workgroup: those of its unit, or of the list.  Of the list the next one is
  // taken while this one's rows load.  (Dealt out in advance, so that also its first block could
  // load early, items of one XCD drift apart and share less of its L2: 2133 us on the 256K
  // share against 1869; and copies under way into the last block's code path cost 4% more.)
  std::conditional_t<ROWS, RowUnit, NoUnit> unit(rows, blockIdx.x);
  const int q_serve = xcd_of_workgroup();
  int q_state = kTakeFirst, turn = 0;
  auto take = [&](int slot) {
    if (w == 0) {
      const int got = take_run_item(a.hdr, kFwdQ, q_serve, q_state);
      if (tid == 0) s_item[slot] = got;
    }
  };
  auto next_item = [&](FwdItem &x) {
    if constexpr (ROWS) {
      return unit.next(rows, x);
    } else {
      const int idx = __builtin_amdgcn_readfirstlane(s_item[turn]);
      if (idx < 0) return false;
      x = load_uniform(a.items + idx);
      turn ^= 1;
      return true;
    }
  };
  // global -> LDS, asynchronous: the K (part 0) or V (part 1) rows of step b of an item.  In
  // the place of a key that none of its rows attends (past the last row, or between the sinks
  // and the window of the first row) one is read that some row does.
  auto issue = [&](const FwdItem &x, int b, int buf, int part) {
    const int kb = step_block(b, x.far, x.gap) * kFwdBN;
    const int last = x.q_loc0 + x.nrows - 1 - kb;   // the last row's key in the block
    const bf16 *base = (part ? a.v : a.k) + ((size_t)(x.sample + kb) * h_kv + x.g) * D;
    const uint32_t ld = lds_addr(smem + buf * S::STAGE + part * S::K_EL) + 1024u * w;
    constexpr uint32_t e = kWaves * 1024u;
    auto copy = [&](const uint32_t (&at)[S::NK]) {
      if constexpr (S::NK == 4) {
        g2l16x4r(base, at[0], at[1], at[2], at[3], ld, ld + e, ld + 2 * e, ld + 3 * e);
      } else {
        g2l16s(base, at[0], ld);
        g2l16s(base, at[1], ld + e);
      }
    };
    if (__builtin_expect(b > x.far && last >= kFwdBN - 1, 1)) {
      copy(k_lane);
    } else {
      // the first row's window begins at `from`, the sinks end at sk
      int from = x.q_loc0 - win.size + 1 - kb, sk = win.sinks - kb;
      asm volatile("" : "+v"(from), "+v"(sk));
      uint32_t at[S::NK];
      static_for<S::NK>([&](auto u) {
        const int r = swu_row<S::KC>(w + kWaves * u, l);
        int key = min(r, last);
        if (key >= sk && key < from) key = from < kFwdBN ? from : sk - 1;
        at[u] = k_lane[u] + 2u * (uint32_t)((key - r) * h_kv * D);
      });
      copy(at);
    }
  };
  // an item's first block, and this lane's query row
  bf16x8 qf[NC];
  auto begin = [&](const FwdItem &x) {
    issue(x, x.kb0, 0, 0);
    issue(x, x.kb0, 0, 1);
    const int first = (w / x.nh) * kRows, count = min(x.nrows - first, kRows);
    if (count > 0) {
      const bf16 *qp = a.q + ((size_t)(x.q_row0 + first + min(ln, count - 1)) * h_q + x.head0 +
                              w % x.nh) * D + 8 * kg;
      static_for<NC>([&](auto c) { qf[c] = *reinterpret_cast<const bf16x8 *>(qp + 16 * c); });
    }
  };

  FwdItem it;
  if constexpr (!ROWS) {
    take(0);
    __syncthreads();
  }
  while (next_item(it)) {
    begin(it);
    if constexpr (!ROWS) take(turn);
    wait_vm_known();   // no wait for Q inside the loop
    __syncthreads();
    const int head = it.head0 + (w % it.nh);
    const int wrow0 = (w / it.nh) * kRows;
    const int wrows = min(max(it.nrows - wrow0, 0), kRows);
    const bool active = wrows > 0;
    const int my_r = active ? min(ln, wrows - 1) : 0;
    const int row = it.q_row0 + wrow0 + my_r;
    const int qloc = it.q_loc0 + wrow0 + my_r;
    const int qmin = it.q_loc0 + wrow0, qlast = qmin + wrows - 1;
    const int kb0 = it.kb0, nkb = it.kb1;   // steps [kb0, nkb)
    // steps of the wave: up to the block of its last row
    const int pend = active ? qlast / kFwdBN + 1 - it.gap : 0;

    f32x16 oacc[NT];
    static_for<NT>([&](auto dt) { oacc[dt] = mfma_zero_c(); });
    float m_run = -INFINITY, l_run = 0.f;
    for (int b = kb0; b < nkb; ++b) {
      const int buf = (b - kb0) & 1;
      const bool more = __builtin_expect(b + 1 < nkb, 1);
      const int kb = step_block(b, it.far, it.gap) * kFwdBN;
      const bf16 *Ks = smem + buf * S::STAGE, *Vs = Ks + S::K_EL;
      // does some row of the wave attend a key of the half that begins at k0?
      auto used = [&](int k0) {
        return b < pend && k0 <= qlast && (k0 + 31 > qmin - win.size || k0 < win.sinks);
      };
      const bool u0 = __builtin_expect(used(kb), 1), u1 = __builtin_expect(used(kb + 32), 1);
      // the next block's K rows after this one's S^T products, its V rows after the softmax
      // (a wave without keys in this block posts both at once)
      if (__builtin_expect(!u0 && !u1, 0)) {
        if (more) {
          issue(it, b + 1, buf ^ 1, 0);
          issue(it, b + 1, buf ^ 1, 1);
        }
      } else {
        f32x16 s[2];
        // S^T, operands read AHEAD products before the one that takes them, also from the
        // first half into the second
        constexpr int AHEAD = D == 64 ? 2 : 4;   // at d = 64 more would spill
        bf16x8 kop[2 * NC];   // product i: half i / NC, chunk i % NC
        const bf16 *kp[2] = {Ks + koff[0], Ks + koff[1]};
        auto rd = [&](auto i) {
          constexpr int t = i / NC, c = i % NC;
          kop[i] = *reinterpret_cast<const bf16x8 *>(kp[c & 1] + 32 * t * D + (c >> 1) * STEP4);
        };
        auto score = [&](auto h_t) {
          constexpr int H = decltype(h_t)::value;
          static_for<NC>([&](auto c) {
            s[H] = mfma32(kop[NC * H + c], qf[c], c == 0 ? mfma_zero_c() : s[H]);
            if constexpr (NC * H + c + AHEAD < 2 * NC)
              rd(std::integral_constant<int, NC * H + c + AHEAD>{});
            __builtin_amdgcn_sched_barrier(0);
          });
        };
        using H0 = std::integral_constant<int, 0>;
        using H1 = std::integral_constant<int, 1>;
        if (__builtin_expect(u0, 1)) {
          static_for<AHEAD>([&](auto i) { rd(i); });
          __builtin_amdgcn_sched_barrier(0);
          score(H0{});
        } else {
          static_for<AHEAD>([&](auto i) { rd(std::integral_constant<int, NC + i>{}); });
          static_for<16>([&](auto r) { s[0][int(r)] = -INFINITY; });
        }
        if (__builtin_expect(u1, 1)) score(H1{});
        else static_for<16>([&](auto r) { s[1][int(r)] = -INFINITY; });
        if (more) issue(it, b + 1, buf ^ 1, 0);
        // Keys that a row does not attend, by their place `at` in the block (less 8 kg): those
        // after the row, at > hi; and from the sinks' end to the window's start, at in
        // [sk, sk + gone).  The empty asm keeps the comparisons in their branch: taken out of it,
        // they need more scalar registers than there are.
        int hi = qloc - kb - 8 * kg;
        if (__builtin_expect(kb + kFwdBN - 1 > qmin, 0)) {
          asm volatile("" : "+v"(hi));
          static_for<2>([&](auto t) {
            static_for<16>([&](auto r) {
              constexpr int at = 32 * t + 16 * (r >> 3) + (r & 7);
              s[t][int(r)] = at > hi ? -INFINITY : s[t][int(r)];
            });
          });
        }
        if (__builtin_expect(kb <= qlast - win.size, 0)) {
          int sk = max(win.sinks - kb - 8 * kg, 0), gone = max(hi - win.size + 1 - sk, 0);
          asm volatile("" : "+v"(sk), "+v"(gone));
          static_for<2>([&](auto t) {
            static_for<16>([&](auto r) {
              constexpr int at = 32 * t + 16 * (r >> 3) + (r & 7);
              s[t][int(r)] = (uint32_t)(at - sk) < (uint32_t)gone ? -INFINITY : s[t][int(r)];
            });
          });
        }
        // P with the running max, which moves only when the block's row sum of P exceeds
        // 256 (as in the causal forward)
        bf16x8 pf[4];
        float ps = 0.f;
        auto expo = [&](float neg_m) {
          ps = 0.f;
          static_for<2>([&](auto t) {
            static_for<16>([&](auto r) {
              const float p = fast_exp2(__builtin_fmaf(s[t][int(r)], a.c2, neg_m));
              ps += p;
              pf[2 * t + (r >> 3)][r & 7] = static_cast<bf16>(p);
            });
          });
        };
        bool move = true;
        if (b > kb0) {
          expo(-m_run);
          move = !(row_sum2(ps) <= 256.f);
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(move) != 0, 0)) {
          float mx = -INFINITY;
          static_for<2>([&](auto t) {
            static_for<16>([&](auto r) { mx = fmaxf(mx, s[t][int(r)]); });
          });
          mx = fmaxf(row_max2(mx) * a.c2, -3.402823466e38f);   // a row may have no key here
          const float alpha = move ? fast_exp2(m_run - mx) : 1.f;
          m_run = move ? mx : m_run;
          l_run *= alpha;
          static_for<NT>([&](auto dt) {
            static_for<16>([&](auto r) { oacc[dt][int(r)] *= alpha; });
          });
          expo(-m_run);
        }
        l_run += ps;
        // O^T += V^T P^T, operands read ahead in the same way
        constexpr int NQ = 2 * NT;   // products of a half
        bf16x8 vop[2 * NQ];
        const bf16 *vp[2] = {Vs + troff[0], Vs + troff[1]};
        auto rt = [&](auto j) {
          constexpr int at = 16 * D * (j / NT) + STEP4 * (j % NT);
          vop[j] = lds_tr16x2(vp[0] + at, vp[1] + at);
        };
        auto add = [&](auto h_t) {
          constexpr int H = decltype(h_t)::value;
          static_for<NQ>([&](auto i) {
            constexpr int j = NQ * H + i;
            oacc[j % NT] = mfma32(vop[j], pf[j / NT], oacc[j % NT]);
            if constexpr (j + AHEAD < 2 * NQ) rt(std::integral_constant<int, j + AHEAD>{});
            __builtin_amdgcn_sched_barrier(0);
          });
        };
        if (__builtin_expect(u0, 1)) static_for<AHEAD>([&](auto j) { rt(j); });
        else static_for<AHEAD>([&](auto j) { rt(std::integral_constant<int, NQ + j>{}); });
        if (more) issue(it, b + 1, buf ^ 1, 1);
        __builtin_amdgcn_sched_barrier(0);
        if (__builtin_expect(u0, 1)) add(H0{});
        if (__builtin_expect(u1, 1)) add(H1{});
      }
      wait_vm();
      __syncthreads();
    }

    const float l_tot = row_sum2(l_run);
    if (active && it.slot >= 0) {
      // a part of a split item: unnormalised O, the running max and the row sum into its
      // partial slot (rows w * 32 + ln)
      if (ln < wrows) {
        float *rec = a.parts + (size_t)it.slot * fwd_part_floats(D);
        float *op = rec + (size_t)(w * kRows + ln) * D + 8 * kg;
        static_for<NT>([&](auto dt) {
          static_for<4>([&](auto q4) {
            constexpr int r0 = 4 * q4;
            *reinterpret_cast<float4 *>(op + 32 * dt + 16 * (q4 >> 1) + 4 * (q4 & 1)) =
                make_float4(oacc[dt][r0], oacc[dt][r0 + 1], oacc[dt][r0 + 2], oacc[dt][r0 + 3]);
          });
        });
        if (kg == 0) {
          rec[(size_t)kFwdPartRows * D + w * kRows + ln] = m_run;
          rec[(size_t)kFwdPartRows * D + kFwdPartRows + w * kRows + ln] = l_tot;
        }
      }
    } else if (active && ln < wrows) {
      const float inv = 1.f / l_tot;
      bf16 *op = a.o + ((size_t)row * h_q + head) * D + 8 * kg;
      static_for<NT>([&](auto dt) {
        static_for<2>([&](auto hh) {
          bf16x8 ov;
          static_for<8>([&](auto i) {
            ov[int(i)] = static_cast<bf16>(oacc[dt][8 * hh + i] * inv);
          });
          *reinterpret_cast<bf16x8 *>(op + 32 * dt + 16 * hh) = ov;
        });
      });
      if (kg == 0)
        a.lse[(size_t)head * a.n_q + row] = (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2;
    }
  }
}

// Merges the parts of single tokens: a workgroup to a (tile, head chunk), whose item it finds
// as the attention kernel does.  Eight columns to a thread; the threads beyond 4 heads x D / 8
// share the parts (`p` mod `kGroups`), each with the recurrence of fwd_combine_kernel, and the
// groups' sums are merged in the same way.
template <int D>
__global__ __launch_bounds__(256) void win_rows_combine_kernel(WinRows a,
                                                               const float *__restrict__ parts,
                                                               bf16 *__restrict__ o,
                                                               float *__restrict__ lse) {
  constexpr size_t PF = fwd_part_floats(D);
  constexpr int C = D / 8, kSlots = 4 * C, kGroups = 256 / kSlots;
  __shared__ float s_acc[kGroups][8][kSlots], s_m[kGroups][kSlots], s_l[kGroups][kSlots];
  RowUnit unit(a, (int64_t)blockIdx.x * a.parts);
  FwdItem it;
  if (!unit.valid || !unit.one_row() || !unit.next(a, it) || it.slot < 0) return;
  // the first part of np: all but the last are as long
  const int slot = threadIdx.x % kSlots, group = threadIdx.x / kSlots;
  const int head_i = min(slot / C, it.nh - 1), col = slot % C * 8;
  const WinTile &t = unit.t;
  const FwdItem whole = win_item(t, it.sample, t.q_begin, t.q_end, 0, 1, it.g, it.head0, it.nh,
                                 a.win);
  const int np = (whole.kb1 + it.kb1 - 1) / it.kb1;
  const float *rec = parts + (size_t)it.slot * PF;
  const int pr = head_i * kRows;   // wave slice head_i, its first row
  float m = -INFINITY;
#pragma unroll 4
  for (int p = group; p < np; p += kGroups)
    m = fmaxf(m, rec[p * PF + (size_t)kFwdPartRows * D + pr]);
  float l = 0.f, acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll 4
  for (int p = group; p < np; p += kGroups) {
    const float *pt = rec + p * PF;
    const float wgt = fast_exp2(pt[(size_t)kFwdPartRows * D + pr] - m);   // finite, both
    l += wgt * pt[(size_t)kFwdPartRows * D + kFwdPartRows + pr];
    const float4 *src = reinterpret_cast<const float4 *>(pt + (size_t)pr * D + col);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 x = src[i];
      acc[4 * i] += wgt * x.x;
      acc[4 * i + 1] += wgt * x.y;
      acc[4 * i + 2] += wgt * x.z;
      acc[4 * i + 3] += wgt * x.w;
    }
  }
  s_m[group][slot] = m;
  s_l[group][slot] = l;
#pragma unroll
  for (int i = 0; i < 8; ++i) s_acc[group][i][slot] = acc[i];
  __syncthreads();
  if (group > 0 || slot / C >= it.nh) return;
#pragma unroll
  for (int u = 1; u < kGroups; ++u) m = fmaxf(m, s_m[u][slot]);
  l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const float wgt = fast_exp2(s_m[u][slot] - m);   // 0 for a group without parts
    l += wgt * s_l[u][slot];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += wgt * s_acc[u][i][slot];
  }
  const float inv = 1.f / l;
  const int head = it.head0 + head_i;
  bf16x8 ov;
#pragma unroll
  for (int i = 0; i < 8; ++i) ov[i] = static_cast<bf16>(acc[i] * inv);
  *reinterpret_cast<bf16x8 *>(o + ((size_t)it.q_row0 * a.h_q + head) * D + col) = ov;
  if (col == 0)
    lse[(size_t)head * a.n_q + it.q_row0] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Head chunks of a tile, and whether a call is one of single tokens.
static int64_t row_chunks(int h_q, int h_kv) { return h_kv * ((h_q / h_kv + 3) / 4); }
static bool row_call(int64_t T, int64_t n_q, int64_t jobs) {
  return n_q <= T && jobs <= kMaxRowJobs;
}
// Key ranges of a single token's item at most, with `slots` for partial results in all.
static int64_t row_cuts(const Window &win, int64_t n_kv, int64_t jobs, int64_t slots) {
  const int64_t steps = win_max_steps(win, n_kv, 1);
  return std::max<int64_t>(
      1, std::min({steps / kRowMinSteps, (int64_t)kRowMaxCuts, slots / jobs}));
}
// A forward's workspace: slots only where its items can be cut, and for single tokens (512 ranges
// fill the card) as many as they can have.
FwdLayout win_fwd_layout(int64_t T, int64_t n, int64_t n_q, int64_t n_kv, int h_q, int h_kv, int d,
                         const Window &win) {
  const int64_t jobs = T * row_chunks(h_q, h_kv);
  int64_t parts = win_may_split(win, n_kv) ? kFwdSplitSlots : 0;
  if (jobs > 0 && row_call(T, n_q, jobs)) {
    const int64_t cuts = row_cuts(win, n_kv, jobs, 512);
    parts = cuts > 1 ? jobs * cuts : 0;
  }
  return fwd_layout(T, n, n_q, n_kv, h_q, h_kv, d, (int)parts);
}

// How a call without a list runs (parts, cuts); false: it has one.
//   * Single tokens, no more Q rows than tiles: one unit for each key range, as many as run at
//     once, two for each CU, and have slots for their partial results (32 / 8 heads, window
//     4096: 32 sequences of 6000 keys 121 us with one for each CU, 98 with two, 105 with four;
//     64 sequences 181, 181 and 191).
//   * Small calls whose items are too short to be cut: as many units as the longest tile that
//     the rows allow has windows, so that none has two (512 tokens, 8 / 2 heads, window 128:
//     16.6 us with a list, 9.9 without).
static bool without_list(WinRows &r, int max_parts, int cus) {
  const int64_t jobs = r.T * r.chunks;
  if (row_call(r.T, r.n_q, jobs)) {
    r.cuts = r.parts =
        (int)row_cuts(r.win, r.n_kv, jobs, std::min<int64_t>(max_parts, 2 * cus));
    return true;
  }
  const int64_t windows = (r.n_q + kRows - 1) / kRows;
  if (win_may_split(r.win, r.n_kv) || jobs > kMaxSmallUnits || jobs * windows > kMaxSmallUnits)
    return false;
  r.parts = (int)windows;
  r.cuts = 1;
  return true;
}

template <int D>
static int launch_win_fwd_d(const WinFwd &a, WinRows rows, const FwdLayout &L, FwdSplit *splits,
                            hipStream_t st, const KernelTimer *tm) {
  using S = WinFwdShape<D>;
  int dev = 0, cus = 256;
  hipGetDevice(&dev);
  hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (without_list(rows, L.max_parts, cus)) {
    if (int rc = reserve_lds<&win_fwd_kernel<D, WinRows>>(S::SMEM)) return rc;
    if (tm) hipEventRecord(tm->begin, st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(win_fwd_kernel<D, WinRows>),
                       dim3((unsigned)(rows.units() + 1)), dim3(kThreads), S::SMEM, st, a, rows);
    if (rows.cuts > 1)
      hipLaunchKernelGGL(win_rows_combine_kernel<D>, dim3((unsigned)(rows.T * rows.chunks)),
                         dim3(256), 0, st, rows, a.parts, a.o, a.lse);
  } else {
    if (int rc = reserve_lds<&win_fwd_kernel<D, NoRows>>(S::SMEM)) return rc;
    const int grid = cus * kWinFwdPerCu<D, false>;
    const int max_parts = win_may_split(a.win, rows.n_kv) ? L.max_parts : 0;
    launch_win_prep_fwd(WinPrep{rows.cu, rows.n, rows.tiles, rows.T, rows.h_q, rows.h_kv, rows.n_q,
                                rows.n_kv, a.win, a.hdr, const_cast<FwdItem *>(a.items),
                                L.max_items, 1, grid, cus * 2, max_parts, splits}, st);
    if (tm) hipEventRecord(tm->begin, st);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(win_fwd_kernel<D, NoRows>), dim3(grid), dim3(kThreads),
                       S::SMEM, st, a, NoRows{});
    if (max_parts > 0)
      launch_fwd_combine(D, splits, a.hdr, a.parts, a.h_q, a.n_q, a.o, a.lse, cus * 4, st);
  }
  if (tm) hipEventRecord(tm->end, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(LIBRA_EHIP, "forward launch failed: %s", hipGetErrorString(e));
  return LIBRA_OK;
}

int launch_win_fwd(const void *q, const void *k, const void *v, const int64_t *cu, int64_t n,
                   const libra_tile_t *tiles, int64_t T, int64_t n_q, int64_t n_kv, int h_q,
                   int h_kv, int d, float scale, void *o, float *lse, void *ws,
                   const FwdLayout &L, hipStream_t st, const KernelTimer *tm, const Window &win) {
  char *W = static_cast<char *>(ws);
  int32_t *hdr = reinterpret_cast<int32_t *>(W + L.hdr);
  const WinFwd a{static_cast<const bf16 *>(q), static_cast<const bf16 *>(k),
                 static_cast<const bf16 *>(v), reinterpret_cast<const FwdItem *>(W + L.items),
                 hdr, h_q, h_kv, n_q, scale * kLog2e, static_cast<bf16 *>(o), lse,
                 reinterpret_cast<float *>(W + L.parts), win};
  const WinRows rows{cu, n, tiles, T, h_q, h_kv, n_q, n_kv, win, hdr,
                     (int)row_chunks(h_q, h_kv), 1, 1};
  auto *splits = reinterpret_cast<FwdSplit *>(W + L.splits);
  return (d == 128 ? launch_win_fwd_d<128> : launch_win_fwd_d<64>)(a, rows, L, splits, st, tm);
}

}  // namespace libra
