"""GPU test of a windowed backward among whose tiles some lie outside the buffers."""
import numpy as np
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from test_gpu_window import blocks, offsets, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h_q,h_kv,d,lengths,window,sinks,good", [
    (4, 2, 64, [700, 133], 90, 4, 4),         # far sinks, items in row ranges
    (3, 1, 128, [500, 200], 64, 0, 9),
    (20, 10, 64, [900, 700], 100, 40, 40),    # whole items
])
def test_skipped_tiles(h_q, h_kv, d, lengths, window, sinks, good):
    """They are counted, and the gradients are those of the other tiles; rows that no good tile
    covers keep what their dQ held."""
    n = sum(lengths)
    tiles = blocks(n, 100, h_q)[:good]
    rows = int((tiles["q_row"] + tiles["q_end"] - tiles["q_begin"]).max()) + 3
    bad = np.zeros(9, dtype=pl.TILE_DTYPE)
    bad["q_begin"], bad["q_end"], bad["head_end"] = 5, 5, h_q         # empty
    bad[0] = (10, 14, rows - 3, 0, 0, h_q, 0, 0, 0, 0)                  # past the Q rows
    bad[1] = (10, 11, 0, 0, 0, h_q + 1, 0, 0, 0, 0)                     # past the heads
    bad[2] = (n - 3, n + 1, 0, 0, 0, h_q, 0, 0, 0, 0)                   # past the keys
    bad[3] = (-1, 2, 0, 0, 0, h_q, 0, 0, 0, 0)                          # before the keys
    bad[4] = (10, 11, -1, 0, 0, h_q, 0, 0, 0, 0)                        # before the Q rows
    every = np.concatenate([bad[:2], tiles[:2], bad[2:5], tiles[2:], bad[5:]])
    say(f"[window skipped] lengths={lengths} heads=({h_q},{h_kv}) d={d} tiles={len(every)}")
    q, k, v, do = tensors(good, rows, n, h_q, h_kv, d)
    pos = torch.cat([ref.positions(tiles), torch.full((3,), -1)])
    cov = torch.cat([ref.coverage(tiles, rows - 3, h_q), torch.zeros((3, h_q), dtype=torch.bool)])
    want = ref.attention(q, k, v, ref.visible(lengths, pos, n, window, sinks), cov, dout=do)
    qd, kd, vd, dod = (x.to(DEV) for x in (q, k, v, do))
    cu, td = offsets(lengths), pl.tiles_to_device(every, DEV)
    mask = dict(window=window, sinks=sinks)
    o, lse = torch.zeros_like(qd), torch.zeros((h_q, rows), device=DEV)
    pl.libra_attn_window_fwd(qd, kd, vd, cu, td, o=o, lse=lse, **mask)
    need = pl.libra_attn_window_workspace_size(len(every), len(lengths), rows, n, h_q, h_kv, d,
                                               True, **mask)
    ws = torch.full((need,), 0xa5, dtype=torch.uint8, device=DEV)
    dq = torch.full_like(qd, 7.0)
    _, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, dq=dq, workspace=ws,
                                         **mask)
    assert pl.libra_attn_skipped_tiles(ws) == len(bad)
    ref.close("dq", dq, want["dq"], cov)
    assert (dq.cpu()[~cov] == 7).all()
    ref.close("dk", dk, want["dk"])
    ref.close("dv", dv, want["dv"])
