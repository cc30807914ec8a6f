"""GPU tests of libra_attn_bwd_ckpt8 besides its gradients at ordinary sizes: what it leaves in
its workspace."""
import numpy as np
import pytest
import torch

import paper_2607_23250_amd as pl
from gpu_util import DEV, say
from test_gpu_window import blocks, offsets, tensors

pytestmark = pytest.mark.gpu


def layer(seed, lengths, tiles, h_q, h_kv, d, window, sinks, change=None, scale=0.0):
    """A layer as it runs: forward on bf16 q, k and v (``change``: of (q, k, v, dout) first), then
    the held tensors; (device q, k, v, dout, o, lse, held, offsets, tiles)."""
    rows = int((tiles["q_row"] + tiles["q_end"] - tiles["q_begin"]).max())
    t = tensors(seed, rows, sum(lengths), h_q, h_kv, d)
    if change:
        t = change(*t)
    q, k, v, do = (x.to(torch.bfloat16).to(DEV) for x in t)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    o, lse = torch.zeros_like(q), torch.zeros((h_q, rows), device=DEV)
    if window:
        pl.libra_attn_window_fwd(q, k, v, cu, td, o=o, lse=lse, window=window, sinks=sinks,
                                 softmax_scale=scale)
    else:
        pl.libra_attn_fwd(q, k, v, cu, td, o=o, lse=lse, softmax_scale=scale)
    return q, k, v, do, o, lse, [pl.libra_ckpt8_pack(x) for x in (q, k, v, o)], cu, td


@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 0), (90, 4)])
def test_skipped_tiles_are_counted(window, sinks):
    """Tiles outside the buffers among good ones: the count in the workspace, which held other
    bytes before, and the same gradients as without them."""
    h_q, h_kv, d, lengths = 4, 2, 64, [700, 133]
    tiles = blocks(833, 200, h_q, 2)
    say(f"[ckpt8 skipped tiles] window={window} sinks={sinks}")
    q, k, _, do, _, lse, held, cu, td = layer(3, lengths, tiles, h_q, h_kv, d, window, sinks)
    bad = np.zeros(7, dtype=pl.TILE_DTYPE)
    bad["q_begin"], bad["q_end"], bad["head_end"] = 5, 5, h_q         # empty
    bad[0] = (10, 11, 833, 0, 0, h_q, 0, 0, 0, 0)                       # past the Q rows
    bad[1] = (10, 11, 0, 0, 0, h_q + 1, 0, 0, 0, 0)                     # past the heads
    bad[2] = (830, 840, 0, 0, 0, h_q, 0, 0, 0, 0)                       # past the keys
    every = np.concatenate([bad[:4], tiles, bad[4:]])
    results = []
    for t, skipped in ((tiles, 0), (every, len(bad))):
        need = pl.libra_attn_bwd_ckpt8_workspace_size(len(t), 2, 833, 833, h_q, h_kv, d,
                                                      window=window, sinks=sinks)
        ws = torch.full((need,), 0xa5, dtype=torch.uint8, device=DEV)
        results.append(pl.libra_attn_bwd_ckpt8(*held, lse, do, cu, pl.tiles_to_device(t, DEV),
                                               window=window, sinks=sinks, workspace=ws))
        assert pl.libra_attn_skipped_tiles(ws) == skipped
    assert all(torch.equal(a, b) for a, b in zip(*results))
