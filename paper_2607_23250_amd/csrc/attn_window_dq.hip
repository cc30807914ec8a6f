// dQ kernel of windowed attention (gfx950).
//
// Its mathematics is the causal dQ kernel's (attn_bwd_dq.hip): S^T = K Q^T, dP^T - D =
// [V | 1] [dO | -D]^T, dS^T = P^T (dP^T - D), dQ^T += K^T dS^T, and the row sums of dS
// correct D for the dK / dV kernel.  The products take the scaled fp16 copies that the dK / dV
// kernel has too (fp16_scale): Q and dO are turned here, those of K and V are there.  So
// dS is rounded to 11 bits, where the causal kernel's bf16 has 8 (dQ of a 32K pack,
// window 1024, against 64 bits: 1.7e-3 of its norm, which is its own rounding to bf16, 2.4e-3
// with dS in bf16).
//
// Its shape is the forward's, because a windowed item is short (19 key blocks with a window
// of 1024): two workgroups of four waves per CU, so that one loads its rows and writes its
// results while the other computes.  Each wave takes both 32-key halves of a block for its
// (query head, 32 rows); halves that no row of the wave attends are passed over.  With one
// workgroup of eight waves per CU, as in the causal kernel, every CU waited about 10 of an
// item's 36 us for its rows: 1146 us for 32K tokens, 32 heads, window 1024, now 879 (870 with
// bf16 products).  Bound by the three products (741 GFLOP there, 843 TFLOP/s) at the clock that
// the card holds under them: the matrix cores are busy half of the cycles, at 1.75 GHz.
//
// The kernel also does what the causal calls leave to a pass of its own over Q, O and dO:
// D = rowsum(dO O), and the records of the dK / dV kernel (see pre_pass in attn_bwd.hip for
// their layout); a split item's first part writes them.
//
// HELD: Q and O in 8 bits (ckpt8.hip); their bf16 values are exact.  LSE is then not that of
// Q and K, so dS can leave the fp16 range: an item whose sums show it is done once more
// (attn_bwd_steps.h), dS as pairs of bf16 numbers.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "attn_bwd_steps.h"
#include "attn_common.h"
#include "attn_win_items.h"
#include "errors.h"

namespace libra {

template <int D>
struct WinDqShape {
  static constexpr int KC = D / 8;            // 16-byte columns of a K / V row
  static constexpr int K_EL = kFwdBN * D;
  static constexpr int STAGE = 2 * K_EL;      // K and V rows of one key block
  static constexpr int NK = kFwdBN * KC / 64 / kWaves;   // wave loads per K (V) tile
  static constexpr size_t SMEM = 2 * STAGE * sizeof(bf16);
  static_assert(NK == 2 || NK == 4, "d = 64 or 128");
};

template <int D, bool HELD>
__global__ __launch_bounds__(kThreads, 2) void win_dq_kernel(WinDq a) {
  using S = WinDqShape<D>;
  constexpr int NC = D / 16, NT = D / 32;
  extern __shared__ __attribute__((aligned(16))) bf16 smem[];
  __shared__ int32_t s_next[2];
  __shared__ int32_t s_wide[2];   // HELD: the item is to be redone
  const int tid = threadIdx.x, l = tid & 63, ln = l & 31, kg = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);   // wave index (uniform)
  const int h_q = a.h_q, h_kv = a.h_kv;
  const Window win = a.win;
  int32_t *hdr = a.hdr;
  const int q_serve = xcd_of_workgroup();
  int q_state = kTakeFirst, turn = 0;
  const float s_q = fp16_scale((uint32_t)hdr[kMaxAbs + 0], false);
  const float s_o = fp16_scale((uint32_t)hdr[kMaxAbs + 1], true);
  const float s_k = fp16_scale((uint32_t)hdr[kMaxAbs + 2], false);
  const float s_v = fp16_scale((uint32_t)hdr[kTopV], true);
  const float s_ov = s_o * s_v, c2s = a.c2 / (s_q * s_k);   // S comes out times s_q s_k, dP s_o s_v
  // P is formed times 16: P |dP - D| is below 2^11 in these units, and small terms stay further
  // from the smallest fp16 numbers.
  constexpr float kUp = 16.f, kLogUp = 4.f;
  const float back = 1.f / (s_k * s_ov * kUp);
  // operand reads and staging as in the forward kernel; half h of a block is 32 h D
  // elements further
  constexpr int STEP4 = S::KC == 16 ? 128 : 256;   // elements from chunk j to chunk j + 4
  const int prow = perm32(ln);
  const int koff[2] = {swu<S::KC>(prow, kg), swu<S::KC>(prow, 2 + kg)};
  int troff[2];
  {
    const int grp = l >> 4, i = (l & 15) >> 2, r = l & 3;
    static_for<2>([&](auto h2) {
      troff[h2] = swu<S::KC>(8 * (grp >> 1) + 4 * h2 + i, 2 * (grp & 1) + (r & 1)) + 4 * (r >> 1);
    });
  }
  uint32_t k_lane[S::NK];
  static_for<S::NK>([&](auto u) {
    const int wl = w + kWaves * u;
    k_lane[u] = 2u * (uint32_t)(swu_row<S::KC>(wl, l) * h_kv * D + 8 * swu_col<S::KC>(wl, l));
  });
  f16x8 ones3;
  static_for<8>([&](auto i) { ones3[int(i)] = f16(kg == 0 && i < 3 ? 1.f : 0.f); });

  if (w == 0) {
    const int got = take_run_item(hdr, kFwdQ, q_serve, q_state);
    if (tid == 0) s_next[0] = got;
  }
  __syncthreads();
  for (;; turn ^= 1) {
    const int idx = __builtin_amdgcn_readfirstlane(s_next[turn]);
    if (idx < 0) break;
    const FwdItem it = load_uniform(a.items + idx);
    const int key0 = it.sample;   // its first key
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

    // global -> LDS, asynchronous: the K (part 0) or V (part 1) rows of step b; keys past
    // the item's last row read that row's key
    auto issue = [&](int b, int buf, int part) {
      const int kb = step_block(b, it.far, it.gap) * kFwdBN;
      const int last = it.q_loc0 + it.nrows - 1 - kb;
      const f16 *base = (part ? a.v16 : a.k16) + ((size_t)(key0 + kb) * h_kv + it.g) * D;
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
      if (__builtin_expect(last >= kFwdBN - 1, 1)) {
        copy(k_lane);
      } else {
        uint32_t at[S::NK];
        static_for<S::NK>([&](auto u) {
          const int r = swu_row<S::KC>(w + kWaves * u, l);
          at[u] = k_lane[u] - 2u * (uint32_t)(max(r - last, 0) * h_kv * D);
        });
        copy(at);
      }
    };
    issue(kb0, 0, 0);
    issue(kb0, 0, 1);

    // Q and dO rows of this lane's query (B operands), LSE log2(e), and -D for dP^T's
    // augmented k-block
    f16x8 qf[NC], of[NC], dneg;
    float dd_q = 0.f, neg_l2 = 0.f;
    if (active) {
      const size_t off = ((size_t)row * h_q + head) * D + 8 * kg;
      const float lv = a.lse[(size_t)head * a.n_q + row];
      bf16x8 qv[NC], ov[NC], dov[NC];
      static_for<NC>([&](auto c) {
        if constexpr (HELD) {
          qv[c] = held8(a.q8, off + 16 * c);
          ov[c] = held8(a.o8, off + 16 * c);
        } else {
          qv[c] = *reinterpret_cast<const bf16x8 *>(a.q + off + 16 * c);
          ov[c] = *reinterpret_cast<const bf16x8 *>(a.o + off + 16 * c);
        }
        dov[c] = *reinterpret_cast<const bf16x8 *>(a.dout + off + 16 * c);
      });
      float dd = 0.f;
      static_for<NC>([&](auto c) {
        static_for<8>([&](auto i) {
          const float x = static_cast<float>(dov[c][int(i)]);
          dd += static_cast<float>(ov[c][int(i)]) * x;
          qf[c][int(i)] = static_cast<f16>(static_cast<float>(qv[c][int(i)]) * s_q);
          of[c][int(i)] = static_cast<f16>(x * s_o);
        });
      });
      dd_q = row_sum2(dd);
      neg_l2 = __builtin_fmaf(-lv, kLog2e, kLogUp);
      if (kb0 == 0 && ln < wrows) {
        // the row's lanes of the extra operands: -LSE / scale and zeros (-D and the copies
        // follow at the end of the item)
        const int r = row % kRows;
        f16 *ag = a.rec + ((size_t)(row / kRows) * h_q + head) * rec_els(D) + 2 * kRows * D +
                  8 * perm32(r);
        f16x8 x;
        if (kg == 0) {
          split3h(-lv / a.scale * (s_q * s_k), x);
          *reinterpret_cast<f16x8 *>(ag) = x;
          // for the merge of the parts
          if (it.slot >= 0)
            a.stats[((size_t)head * (a.nq_pad / kRows) + row / kRows) * 2 * kRows + kRows + r] =
                dd_q;
        } else {
          static_for<8>([&](auto i) { x[int(i)] = f16(0.f); });
          *reinterpret_cast<f16x8 *>(ag + kAugEl / 4) = x;
          *reinterpret_cast<f16x8 *>(ag + 3 * (kAugEl / 4)) = x;
        }
      }
    }
    split3h(kg == 0 ? -dd_q * s_ov : 0.f, dneg);
    if constexpr (HELD)
      if (tid == 0) s_wide[turn] = 0;
    // the next item, while this one's rows are under way
    if (w == 0) {
      const int got = take_run_item(hdr, kFwdQ, q_serve, q_state);
      if (tid == 0) s_next[turn ^ 1] = got;
    }
    f32x16 acc[NT];
    static_for<NT>([&](auto dt) { acc[dt] = mfma_zero_c(); });
    float d_run = 0.f;      // this lane's sum over its keys, of dS (HELD: of P)
    wait_vm_known();   // no wait for the rows inside the loop
    __syncthreads();

    // the item's steps; WIDE: dS in the range of fp32
    auto walk = [&](auto wide_t) {
      constexpr bool WIDE = decltype(wide_t)::value;
      for (int b = kb0; b < nkb; ++b) {
        const int buf = (b - kb0) & 1;
        const bool more = __builtin_expect(b + 1 < nkb, 1);
        const int kb = step_block(b, it.far, it.gap) * kFwdBN;
        const bf16 *Ks = smem + buf * S::STAGE;
        f16x8 dsf[2][2];   // dS^T of the halves (B operands, two 16-key chunks)
        bf16x8 dsw[2][2];  // WIDE: dS^T of one half and its rest
        // Half H of the block: S^T, dP^T - D (with the exponentials of P^T on the VALU), dS^T.
        // copy: posts the next block's K rows after S^T, its V rows after dP^T.
        auto half = [&](auto h_t, bool copy) {
          constexpr int H = decltype(h_t)::value;
          constexpr int AHEAD = 4;
          const bf16 *kp[2] = {Ks + koff[0] + 32 * H * D, Ks + koff[1] + 32 * H * D};
          f32x16 sa, pa;
          f16x8 op[2 * NC];   // MFMA i < NC: S^T from K; NC + c: dP^T from V
          auto rd = [&](auto i) {
            constexpr int kind = i / NC, c = i % NC;
            op[i] = *reinterpret_cast<const f16x8 *>(kp[c & 1] + kind * S::K_EL + (c >> 1) * STEP4);
          };
          static_for<AHEAD>([&](auto i) { rd(i); });
          __builtin_amdgcn_sched_barrier(0);
          static_for<NC>([&](auto c) {
            sa = mfma32h(op[c], qf[c], c == 0 ? mfma_zero_c() : sa);
            rd(std::integral_constant<int, c + AHEAD>{});
            __builtin_amdgcn_sched_barrier(0);
          });
          if (copy) issue(b + 1, buf ^ 1, 0);
          // keys that a row does not attend, as in the forward
          const int k0 = kb + 32 * H;
          int hi = qloc - k0 - 8 * kg;
          if (__builtin_expect(k0 + 31 > qmin, 0)) {
            asm volatile("" : "+v"(hi));
            static_for<16>([&](auto r) {
              constexpr int at = 16 * (r >> 3) + (r & 7);
              sa[int(r)] = at > hi ? -INFINITY : sa[int(r)];
            });
          }
          if (__builtin_expect(k0 <= qlast - win.size, 0)) {
            int sk = max(win.sinks - k0 - 8 * kg, 0), gone = max(hi - win.size + 1 - sk, 0);
            asm volatile("" : "+v"(sk), "+v"(gone));
            static_for<16>([&](auto r) {
              constexpr int at = 16 * (r >> 3) + (r & 7);
              sa[int(r)] = (uint32_t)(at - sk) < (uint32_t)gone ? -INFINITY : sa[int(r)];
            });
          }
          __builtin_amdgcn_sched_barrier(0);
          pa = mfma32h(ones3, dneg, mfma_zero_c());
          static_for<NC>([&](auto c) {
            pa = mfma32h(op[NC + c], of[c], pa);
            if constexpr (NC + c + AHEAD < 2 * NC)
              rd(std::integral_constant<int, NC + c + AHEAD>{});
            // P^T = exp2(S^T c2 - LSE log2 e), 16 / NC elements per product
            static_for<16 / NC>([&](auto e) {
              constexpr int r = (16 / NC) * c + e;
              float p = fast_exp2(__builtin_fmaf(sa[r], c2s, neg_l2));
              asm volatile("" : "+v"(p));   // stays in its slot
              sa[r] = p;                    // P^T in place
            });
            __builtin_amdgcn_sched_barrier(0);
          });
          if (copy) issue(b + 1, buf ^ 1, 1);
          static_for<16>([&](auto r) {
            const float ds = sa[int(r)] * pa[int(r)];
            d_run += HELD ? sa[int(r)] : ds;
            if constexpr (WIDE) {
              const bf16 x = static_cast<bf16>(ds);
              dsw[0][r >> 3][r & 7] = x;
              dsw[1][r >> 3][r & 7] = static_cast<bf16>(ds - static_cast<float>(x));
            } else {
              dsf[H][r >> 3][r & 7] = static_cast<f16>(ds);
            }
          });
        };
        // dQ^T += K^T dS^T of half H
        auto add = [&](auto h_t) {
          constexpr int H = decltype(h_t)::value, NQ = 2 * NT, TA = 3;
          const bf16 *kt[2] = {Ks + troff[0] + 32 * H * D, Ks + troff[1] + 32 * H * D};
          f16x8 tp[NQ];
          auto rt = [&](auto j) {
            constexpr int at = 16 * D * (j / NT) + STEP4 * (j % NT);
            tp[j] = lds_tr16x2h(reinterpret_cast<const f16 *>(kt[0]) + at,
                                reinterpret_cast<const f16 *>(kt[1]) + at);
          };
          if constexpr (WIDE) {
            static_for<NQ>([&](auto j) {
              rt(j);
              bf16x8 x;
              static_for<8>([&](auto i) {
                x[int(i)] = static_cast<bf16>(static_cast<float>(tp[j][int(i)]));
              });
              static_for<2>([&](auto rest) {
                acc[j % NT] = mfma32(x, dsw[rest][j / NT], acc[j % NT]);
              });
            });
            return;
          }
          static_for<TA>([&](auto j) { rt(j); });
          static_for<NQ>([&](auto j) {
            acc[j % NT] = mfma32h(tp[j], dsf[H][j / NT], acc[j % NT]);
            if constexpr (j + TA < NQ) rt(std::integral_constant<int, j + TA>{});
            __builtin_amdgcn_sched_barrier(0);
          });
        };
        using H0 = std::integral_constant<int, 0>;
        using H1 = std::integral_constant<int, 1>;
        // does some row of the wave attend a key of the half that begins at k0?
        auto used = [&](int k0) {
          return b < pend && k0 <= qlast && (k0 + 31 > qmin - win.size || k0 < win.sinks);
        };
        const bool u0 = used(kb), u1 = used(kb + 32);
        // one place for each: accumulators that came from several would be copied
        if (__builtin_expect(u0, 1)) half(H0{}, more);
        else if (more) issue(b + 1, buf ^ 1, 0), issue(b + 1, buf ^ 1, 1);
        if constexpr (WIDE)
          if (u0) add(H0{});
        if (__builtin_expect(u1, 1)) half(H1{}, false);
        if constexpr (!WIDE)
          if (__builtin_expect(u0, 1)) add(H0{});
        if (__builtin_expect(u1, 1)) add(H1{});
        wait_vm();
        __syncthreads();
      }
    };
    walk(std::false_type{});
    if constexpr (HELD) {
      // a row whose P is small altogether would keep too few bits
      const float p_sum = row_sum2(d_run);
      const bool out = active && (not_finite(acc) || (p_sum > 0.f && p_sum < kUp / 1024));
      if (__builtin_amdgcn_ballot_w64(out) && l == 0) s_wide[turn] = 1;
      __syncthreads();
      if (__builtin_expect(s_wide[turn], 0)) {
        issue(kb0, 0, 0);
        issue(kb0, 0, 1);
        static_for<NT>([&](auto dt) { acc[dt] = mfma_zero_c(); });
        wait_vm();
        __syncthreads();
        walk(std::true_type{});
      }
    }

    const float d_sum = HELD ? 0.f : row_sum2(d_run);   // times 16 s_o s_v; HELD: not needed
    if (active && it.slot >= 0) {
      // a part of a split item: unscaled fp32 dQ and its sum of dS, merged by
      // bwd_dq_combine_kernel
      if (ln < wrows) {
        float *part = a.parts + (size_t)it.slot * fwd_part_floats(D);
        float *op = part + (size_t)(w * kRows + ln) * D + 8 * kg;
        static_for<NT>([&](auto dt) {
          static_for<4>([&](auto q4) {
            constexpr int r0 = 4 * q4;
            *reinterpret_cast<float4 *>(op + 32 * dt + 16 * (q4 >> 1) + 4 * (q4 & 1)) =
                make_float4(acc[dt][r0] * back, acc[dt][r0 + 1] * back, acc[dt][r0 + 2] * back,
                            acc[dt][r0 + 3] * back);
          });
        });
        if (kg == 0) part[(size_t)kFwdPartRows * D + w * kRows + ln] = d_sum / (s_ov * kUp);
      }
    } else if (active && ln < wrows) {
      bf16 *op = a.dq + ((size_t)row * h_q + head) * D + 8 * kg;
      static_for<NT>([&](auto dt) {
        static_for<2>([&](auto hh) {
          bf16x8 x;
          static_for<8>([&](auto i) {
            x[int(i)] = static_cast<bf16>(acc[dt][8 * hh + i] * (a.scale * back));
          });
          *reinterpret_cast<bf16x8 *>(op + 32 * dt + 16 * hh) = x;
        });
      });
    }
    if (active && kb0 == 0 && ln < wrows) {
      // this row of its record
      f16 *rp = a.rec + ((size_t)(row / kRows) * h_q + head) * rec_els(D);
      const int r = row % kRows;
      static_for<NC>([&](auto c) {
        *reinterpret_cast<f16x8 *>(rp + rec_at(r, 2 * c + kg)) = qf[c];
        *reinterpret_cast<f16x8 *>(rp + kRows * D + rec_at(r, 2 * c + kg)) = of[c];
      });
      if (kg == 0 && it.slot < 0) {   // D, corrected (the merge does it for parts)
        f16x8 x;
        split3h(-(dd_q * s_ov + d_sum / kUp), x);
        *reinterpret_cast<f16x8 *>(rp + 2 * kRows * D + kAugEl / 2 + 8 * perm32(r)) = x;
      }
    }
  }
}

template <int D, bool HELD>
static int launch(const WinDq &a, int cus, hipStream_t st) {
  if (int rc = reserve_lds<&win_dq_kernel<D, HELD>>(WinDqShape<D>::SMEM)) return rc;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(win_dq_kernel<D, HELD>), dim3(cus * kWinDqPerCu),
                     dim3(kThreads), WinDqShape<D>::SMEM, st, a);
  return LIBRA_OK;
}
int launch_win_dq(int d, const WinDq &a, int cus, hipStream_t st) {
  const bool held = a.q8.q != nullptr;
  return d == 128 ? (held ? launch<128, true> : launch<128, false>)(a, cus, st)
                  : (held ? launch<64, true> : launch<64, false>)(a, cus, st);
}

}  // namespace libra
