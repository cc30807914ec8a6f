"""GPU test of gradients of tensors so small that products of dO and V, or of the scales that bring
them to fp16, leave fp32: causal, windowed and from checkpoints, under the bounds of window_ref.py
and grad_bounds.py (which let go what lies below the smallest normal fp32 number)."""
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from grad_bounds import gradients
from test_gpu_window import blocks, offsets, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("of_do,of_v", [(-70, -70), (-60, -61), (-100, -20), (-20, -100),
                                        (-115, 3), (-40, -40)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3)])
def test_small_tensors(of_do, of_v, window, sinks, monkeypatch):
    h_q, h_kv, d, lengths = 4, 2, 64, [500, 120]
    say(f"[tiny] dO * 2^{of_do} V * 2^{of_v} window={window}")
    n = sum(lengths)
    tiles = blocks(n, 128, h_q, 2)
    q, k, v, do = tensors(7, n, n, h_q, h_kv, d)
    v, do = v * 2.0 ** of_v, do * 2.0 ** of_do
    pairs = (ref.visible(lengths, ref.positions(tiles), n, window, sinks),
             torch.ones((n, h_q), dtype=torch.bool))
    qd, kd, vd, dod = (x.to(DEV) for x in (q, k, v, do))
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    if window:
        mask = dict(window=window, sinks=sinks)
        o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
        got = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask)
    else:
        o, lse = pl.libra_attn_fwd(qd, kd, vd, cu, td)
        got = pl.libra_attn_bwd(qd, kd, vd, o, lse, dod, cu, td)
    want = gradients(monkeypatch, q, k, v, do, pairs, d ** -0.5, lse.cpu())
    for what, x in zip(("dq", "dk", "dv"), got):
        ref.close(what, x, want[what])
    held = [pl.libra_ckpt8_pack(x) for x in (qd, kd, vd, o)]
    q8, k8, v8, o8 = (pl.libra_ckpt8_unpack(*x, dtype=torch.float32).cpu() for x in held)
    want = gradients(monkeypatch, q8, k8, v8, do, pairs, d ** -0.5, lse.cpu(), (o8, lse.cpu()))
    got = pl.libra_attn_bwd_ckpt8(*held, lse, dod, cu, td, window=window, sinks=sinks)
    for what, x in zip(("dq", "dk", "dv"), got):
        ref.close(what, x, want[what])
