"""GPU tests of attention gradients under a caller's softmax_scale, from very small ones (near
uniform attention) to ones that leave a row one key: causal, windowed and from checkpoints,
against float64 under the bounds of window_ref.py and grad_bounds.py."""
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from grad_bounds import gradients
from test_gpu_window import blocks, offsets, tensors

pytestmark = pytest.mark.gpu

SHAPES = {   # lengths, tiles, heads, d, window, sinks
    "causal": ([600, 90], blocks(690, 128, 4, 2), (4, 2), 64, 0, 0),
    "window": ([500, 190], blocks(690, 200, 4), (4, 1), 128, 90, 2),
    "far_sinks": ([1100], blocks(1100, 256, 6, 2), (6, 2), 64, 130, 5),
}


@pytest.mark.parametrize("scale,size", [(1.5, 1.0), (0.5, 4.0), (0.02, 1.0), (1e-3, 1.0),
                                        (3e-4, 1.0), (1e-5, 1.0), (1e-7, 1.0), (1e-5, 300.0)])
@pytest.mark.parametrize("name", SHAPES)
def test_gradients(name, scale, size, monkeypatch):
    lengths, tiles, (h_q, h_kv), d, window, sinks = SHAPES[name]
    say(f"[scale {name}] softmax_scale={scale} size={size}")
    n = sum(lengths)
    q, k, v, do = tensors(11, n, n, h_q, h_kv, d)
    q, k = q * size, k * size
    pairs = (ref.visible(lengths, ref.positions(tiles), n, window, sinks),
             ref.coverage(tiles, n, h_q))
    # LSE / scale has to fit fp16 as well, so q and k are held lower: by 2^ceil(t / 2) at most
    down = max(1.0, 2 * (22.0 / scale / 32768) ** 0.5)
    exact = ref.attention(q, k, v, *pairs, scale=scale)["lse"][0]
    want = gradients(monkeypatch, q, k, v, do, pairs, scale, exact, down=down)
    qd, kd, vd, dod = (x.to(DEV) for x in (q, k, v, do))
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    if window:
        mask = dict(window=window, sinks=sinks, softmax_scale=scale)
        o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
        got = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask)
    else:
        o, lse = pl.libra_attn_fwd(qd, kd, vd, cu, td, softmax_scale=scale)
        got = pl.libra_attn_bwd(qd, kd, vd, o, lse, dod, cu, td, softmax_scale=scale)
    torch.cuda.synchronize()
    for what, x in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *got)):
        if what == "lse":
            ref.close(what, x, (exact, want["lse"][1]))
        else:
            ref.close(what, x, want[what])
    held = [pl.libra_ckpt8_pack(x) for x in (qd, kd, vd, o)]
    q8, k8, v8, o8 = (pl.libra_ckpt8_unpack(*x, dtype=torch.float32).cpu() for x in held)
    want = gradients(monkeypatch, q8, k8, v8, do, pairs, scale, lse.cpu(), (o8, lse.cpu()), down)
    got = pl.libra_attn_bwd_ckpt8(*held, lse, dod, cu, td, window=window, sinks=sinks,
                                  softmax_scale=scale)
    for what, x in zip(("dq", "dk", "dv"), got):
        ref.close(what, x, want[what])
