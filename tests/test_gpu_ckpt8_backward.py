"""GPU tests of libra_attn_bwd_ckpt8 besides its gradients at ordinary sizes: what it leaves in
its workspace, scores that the 8 bits move far, and dQ items cut into key ranges."""
import numpy as np
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from grad_bounds import gradients
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


def outliers(size):
    """q and k with one large channel each: it sets the unit of its 32 elements, so the others
    round coarsely, and meets them in the scores."""
    def change(q, k, v, do):
        q, k = 2 * q, 2 * k
        q[..., 3] += size
        k[..., 17] += size
        return q, k, v, do
    return change


LARGE = {   # seed, lengths, tiles, heads, d, window, sinks; items cut into row ranges or whole
    "causal_cut": (6, [700, 60], blocks(760, 128, 4, 2), (4, 2), 128, 0, 0),
    "causal_cut_odd": (10, [500], blocks(500, 500, 3), (3, 1), 64, 0, 0),
    "causal_whole": (11, [140] * 12, blocks(1680, 512, 8), (8, 4), 64, 0, 0),
    "window_cut": (6, [900, 77], blocks(977, 300, 4), (4, 1), 64, 120, 0),
    "window_cut_odd_far": (5, [1300], blocks(1300, 256, 3), (3, 1), 128, 100, 40),
    "window_whole_far": (10, [1500, 200], blocks(1700, 512, 20, 2), (20, 10), 64, 150, 8),
}


@pytest.mark.parametrize("name", LARGE)
def test_large_scores(name, monkeypatch):
    """Scores of some hundreds and outlier channels: the rounding of q and k moves scores by more
    than 11, so that P = exp(S - LSE) passes what fp16 holds, and dV and dK with it."""
    seed, lengths, tiles, (h_q, h_kv), d, window, sinks = LARGE[name]
    say(f"[ckpt8 large scores {name}] lengths={lengths} heads=({h_q},{h_kv}) d={d} "
        f"window={window} sinks={sinks}")
    _, _, _, do, o, lse, held, cu, td = layer(seed, lengths, tiles, h_q, h_kv, d, window,
                                              sinks, outliers(150.0))
    q8, k8, v8, o8 = (pl.libra_ckpt8_unpack(*x, dtype=torch.float32).cpu() for x in held)
    lse_h, do_h = lse.cpu(), do.cpu()
    n = sum(lengths)
    pairs = (ref.visible(lengths, ref.positions(tiles), n, window, sinks),
             ref.coverage(tiles, n, h_q))
    want = gradients(monkeypatch, q8, k8, v8, do_h, pairs, d ** -0.5, lse_h, (o8, lse_h))
    # the largest P of each key, and of the far rows of sinks
    top = torch.stack([(torch.exp((q8[:, h].double() @ k8[:, h * h_kv // h_q].double().T)
                                  * d ** -0.5 - lse_h[h, :, None].double()) * pairs[0])
                       for h in range(h_q)]).amax(0)
    assert 65504 < float(top.max()) < 1e30
    if sinks:
        assert float(top[window + sinks:lengths[0], :sinks].max()) > 65504
    results = []
    for accumulate in (False, True, False):
        results.append(pl.libra_attn_bwd_ckpt8(*held, lse, do, cu, td, window=window, sinks=sinks,
                                               accumulate=accumulate))
        for what, got in zip(("dq", "dk", "dv"), results[-1]):
            value, bound = want[what]
            ref.close(what, got, (value, bound + 2.0 ** -23 * value.abs()))
    assert all(torch.equal(a, b) for a, b in zip(results[0], results[2]))


CUT = {   # lengths, tiles, heads, d, window, sinks: few rows late in a long sample
    "causal": ([40, 6000], blocks(6040, 512, 4, 2, [(5600, 6000)]), (4, 2), 128, 0, 0),
    "causal_d64": ([5100], blocks(5100, 300, 3, ranges=[(4700, 5100)]), (3, 1), 64, 0, 0),
    "window": ([2600, 40], blocks(2640, 300, 4, 2), (4, 2), 64, 2500, 3),
    "window_far": ([7, 4000], blocks(4007, 512, 2, ranges=[(3500, 4007)]), (2, 1), 128, 1800, 5),
}


@pytest.mark.parametrize("name", CUT)
def test_cut_dq_items(name, monkeypatch):
    """dQ items cut into key ranges: the parts' merge takes D as it is, whatever the parts' sums
    of dS, and (windowed) a cut item's first part writes the records of held q and dout.  With
    large channels those sums are not near zero: D corrected by them puts dK 8 bounds off."""
    lengths, tiles, (h_q, h_kv), d, window, sinks = CUT[name]
    say(f"[ckpt8 cut dQ {name}] lengths={lengths} heads=({h_q},{h_kv}) d={d} window={window}")
    _, _, _, do, _, lse, held, cu, td = layer(5, lengths, tiles, h_q, h_kv, d, window, sinks,
                                            outliers(30.0))
    rows, n_kv = do.shape[0], sum(lengths)
    need = pl.libra_attn_bwd_ckpt8_workspace_size(len(tiles), len(lengths), rows, n_kv, h_q, h_kv,
                                                  d, window=window, sinks=sinks)
    ws = pl.alloc_workspace(need, DEV)
    got = pl.libra_attn_bwd_ckpt8(*held, lse, do, cu, td, window=window, sinks=sinks,
                                  workspace=ws)
    assert int(ws[:4096].view(torch.int32)[60]) > 0   # items that were cut
    q8, k8, v8, o8 = (pl.libra_ckpt8_unpack(*x, dtype=torch.float32).cpu() for x in held)
    pairs = (ref.visible(lengths, ref.positions(tiles), n_kv, window, sinks),
             ref.coverage(tiles, rows, h_q))
    want = gradients(monkeypatch, q8, k8, v8, do.cpu(), pairs, d ** -0.5, lse.cpu(),
                     (o8, lse.cpu()))
    for what, x in zip(("dq", "dk", "dv"), got):
        ref.close(what, x, want[what])
