"""GPU test of windowed gradients where far samples would be so many, and sinks too, that only the
longer ones are taken as such."""
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from test_gpu_window import blocks, offsets, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,window,sinks,far_rows", [
    ([270] * 14 + [1500, 5, 280, 281, 277], 8, 1024, 352),   # 6123 // 17 - 8
    ([265] * 22, 8, 1000, 334),                              # none is far
    ([300] * 30 + [2000], 8, 600, 399),                      # 11000 // 27 - 8
])
def test_fewer_far_samples(lengths, window, sinks, far_rows):
    h_q, h_kv, d, n = 16, 8, 64, sum(lengths)
    per = h_kv * (-(-sinks // 32))
    assert far_rows == n // (4096 // per + 1) - window   # the line, past the usual 256
    say(f"[fewer far samples] lengths={lengths[:1]}.. {len(lengths)} samples, {n} keys")
    tiles = blocks(n, 512, h_q)
    pos = ref.positions(tiles)
    qd, kd, vd, dod = (x.to(DEV) for x in tensors(n, n, n, h_q, h_kv, d))
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    mask = dict(window=window, sinks=sinks)
    need = pl.libra_attn_window_workspace_size(len(tiles), len(lengths), n, n, h_q, h_kv, d, True,
                                               **mask)
    ws = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
    o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
    dq, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, workspace=ws[:need],
                                          **mask)
    assert bool((ws[need:] == 0xa5).all())
    want = ref.attention(qd, kd, vd, ref.visible(lengths, pos, n, window, sinks),
                         torch.ones((n, h_q), dtype=torch.bool), dout=dod)
    for what, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        ref.close(what, x, want[what])
