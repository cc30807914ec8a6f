"""GPU test that windowed forwards stay inside the workspace that their size function asks for:
those of single tokens, with few and with many key ranges, small ones without a list, and ones
whose list's items are whole or cut."""
import numpy as np
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from test_gpu_window import blocks, offsets, tensors, tile_list

pytestmark = pytest.mark.gpu


def newest(lengths, h_q):
    return tile_list([(int(e) - 1, int(e), 0, h_q) for e in np.cumsum(lengths)])


@pytest.mark.parametrize("name,lengths,tiles,heads,d,window", [
    ("one token", [2500], newest([2500], 8), (8, 2), 64, 1024),
    ("one token of a long cache", [20001], newest([20001], 2), (2, 1), 128, 30000),
    ("one token, one block", [40], newest([40], 4), (4, 4), 64, 100),
    ("tokens", [900, 70, 3000, 1], newest([900, 70, 3000, 1], 16), (16, 2), 128, 2000),
    ("many tokens", [130] * 600, newest([130] * 600, 4), (4, 2), 64, 4096),
    ("small", [512], blocks(512, 256, 8), (8, 2), 64, 128),
    ("list", [5000, 300], blocks(5300, 1024, 8, 2), (8, 2), 64, 300),
    ("cut list", [3000], blocks(3000, 512, 2), (2, 1), 128, 2500),
])
def test_forward(name, lengths, tiles, heads, d, window):
    (h_q, h_kv), n, mask = heads, sum(lengths), dict(window=window, sinks=4)
    pos = ref.positions(tiles)
    say(f"[window workspace] {name}")
    q, k, v, _ = tensors(n, len(pos), n, h_q, h_kv, d)
    sizes = (len(tiles), len(lengths), len(pos), n, h_q, h_kv, d)
    need = pl.libra_attn_window_workspace_size(*sizes, False, **mask)
    ws = torch.full((need + 65536,), 0xa5, dtype=torch.uint8, device=DEV)
    o, lse = pl.libra_attn_window_fwd(q.to(DEV), k.to(DEV), v.to(DEV), offsets(lengths),
                                      pl.tiles_to_device(tiles, DEV), workspace=ws[:need], **mask)
    assert bool((ws[need:] == 0xa5).all())
    want = ref.attention(q, k, v, ref.visible(lengths, pos, n, **mask),
                         ref.coverage(tiles, len(pos), h_q)) if n < 10000 else None
    if want is None:   # by the last 1000 keys' samples, or the only one's
        a = 0 if len(lengths) == 1 else n - 130 * 8
        rows = slice(0, 1) if a == 0 else slice(len(pos) - 8, None)
        want = ref.attention(q[rows], k[a:], v[a:], ref.visible(
            lengths if a == 0 else [130] * 8, pos[rows] - a, n - a, **mask),
            torch.ones((len(pos[rows]), h_q), dtype=torch.bool))
        o, lse = o[rows], lse[:, rows]
    ref.close("o", o, want["o"])
    ref.close("lse", lse, want["lse"])
