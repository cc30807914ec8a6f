"""GPU tests of windowed attention (libra_attn_window_fwd / libra_attn_window_bwd) against
dense attention in float64; the bounds are derived in window_ref.py."""
import numpy as np
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say

pytestmark = pytest.mark.gpu


def offsets(lengths):
    cu = np.zeros(len(lengths) + 1, dtype=np.int64)
    cu[1:] = np.cumsum(lengths)
    return torch.from_numpy(cu).to(DEV)


def tile_list(spans):
    """Tiles (q_begin, q_end, head_begin, head_end) with their Q rows one after another; spans
    of the same positions share rows."""
    rows, out, at = {}, np.zeros(len(spans), dtype=pl.TILE_DTYPE), 0
    for i, (b, e, hb, he) in enumerate(spans):
        if (b, e) not in rows:
            rows[b, e] = at
            at += e - b
        out[i] = (b, e, rows[b, e], 0, hb, he, 0, 0, 0, i)
    return out


def blocks(total, B, h_q, H=1, ranges=None):
    w = h_q // H
    return tile_list([(b, min(b + B, y), s * w, (s + 1) * w) for x, y in (ranges or [(0, total)])
                      for b in range(x, y, B) for s in range(H)])


def tensors(seed, n_q, n_kv, h_q, h_kv, d, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [(torch.randn((n, h, d), generator=gen) * size).to(torch.bfloat16)
            for n, h in ((n_q, h_q), (n_kv, h_kv), (n_kv, h_kv), (n_q, h_q))]


# (lengths, tiles, heads, d, window, sinks)
def _cases():
    yield "one_key", [1], blocks(1, 1, 4), (4, 4), 64, 1, 0
    yield "self_only", [300], blocks(300, 128, 2), (2, 1), 64, 1, 0
    yield "self_and_first", [300, 5], blocks(305, 128, 2), (2, 1), 128, 1, 1
    yield "window_2", [200, 61, 1, 1, 40], blocks(303, 100, 6), (6, 2), 64, 2, 3
    yield "block_edges", [64, 128, 63, 65, 257], blocks(577, 64, 8, 2), (8, 2), 128, 64, 0
    yield "window_63", [700], blocks(700, 700, 4), (4, 2), 64, 63, 64
    yield "window_65", [700], blocks(700, 333, 4, 4), (4, 1), 128, 65, 1
    yield "sinks_65", [900, 100], blocks(1000, 256, 4), (4, 4), 64, 100, 65
    yield "far_sinks", [1500], blocks(1500, 256, 4, 2), (4, 2), 128, 200, 4
    yield "far_many_sinks", [1700, 90], blocks(1790, 600, 3), (3, 1), 64, 129, 300
    yield "far_1024_sinks", [2100], blocks(2100, 512, 2), (2, 1), 64, 40, 1024
    yield "wide", [1000, 300], blocks(1300, 256, 8), (8, 2), 128, 5000, 2
    yield "one_head", [800], blocks(800, 200, 1), (1, 1), 128, 130, 3
    yield "five_heads", [500, 77], blocks(577, 577, 5), (5, 1), 64, 90, 2
    yield "sixteen_heads", [600], blocks(600, 99, 16, 4), (16, 2), 64, 77, 5
    # tiles in no order, of single rows and of part of a KV group's heads
    yield "scattered", [900, 200], tile_list(
        [(1000, 1100, 0, 3), (17, 18, 0, 4), (600, 731, 1, 2), (899, 901, 2, 4), (300, 340, 3, 4)]
    ), (4, 1), 64, 50, 7
    # a context-parallel share: rows at both ends of a long sample
    yield "share", [2000], blocks(2000, 128, 4, 2, [(0, 200), (1800, 2000)]), (4, 2), 128, 150, 4
    yield "deep_tile", [30, 2500], tile_list([(2300, 2420, 0, 2)]), (4, 2), 64, 300, 33
    # items long enough to be cut into key ranges
    yield "cut", [2600, 40], blocks(2640, 300, 4, 2), (4, 2), 128, 2500, 3
    yield "cut_3_heads", [7, 1900], blocks(1907, 512, 3), (3, 1), 64, 1800, 0
    # rows past the last sample
    yield "past_the_end", [100, 150], blocks(320, 64, 2), (2, 2), 64, 30, 2


CASES = {c[0]: c[1:] for c in _cases()}


@pytest.mark.parametrize("name", CASES)
def test_forward_and_backward(name):
    lengths, tiles, (h_q, h_kv), d, window, sinks = CASES[name]
    say(f"[window {name}] lengths={lengths} tiles={len(tiles)} heads=({h_q},{h_kv}) d={d} "
        f"window={window} sinks={sinks}")
    pos = ref.positions(tiles)
    n_q, n_kv = len(pos), max(sum(lengths), int(tiles["q_end"].max()))
    q, k, v, do = tensors(len(name), n_q, n_kv, h_q, h_kv, d)
    cov = ref.coverage(tiles, n_q, h_q)
    ok = ref.visible(lengths, pos, n_kv, window, sinks)
    live = cov & ok.any(1)[:, None]
    want = ref.attention(q, k, v, ok, cov, dout=do)
    qd, kd, vd, dod = (t.to(DEV) for t in (q, k, v, do))
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    mask = dict(window=window, sinks=sinks)
    # outputs outside the covered pairs stay as they were
    o = torch.full_like(qd, 7.0)
    lse = torch.full((h_q, n_q), 7.0, device=DEV)
    pl.libra_attn_window_fwd(qd, kd, vd, cu, td, o=o, lse=lse, **mask)
    torch.cuda.synchronize()
    ref.close("o", o, want["o"], live)
    ref.close("lse", lse, want["lse"], live.T)
    assert (o.cpu()[~live] == 7).all() and (lse.cpu()[~live.T] == 7).all()
    dq = torch.full_like(qd, 7.0)
    _, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, dq=dq, **mask)
    torch.cuda.synchronize()
    ref.close("dq", dq, want["dq"], live)
    assert (dq.cpu()[~live] == 7).all()
    ref.close("dk", dk, want["dk"])
    ref.close("dv", dv, want["dv"])
    # added to what is there
    dk32, dv32 = torch.full(kd.shape, 2.0, device=DEV), torch.full(kd.shape, -1.0, device=DEV)
    pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, dq=dq, dk=dk32, dv=dv32,
                             accumulate=True, **mask)
    torch.cuda.synchronize()
    # the sum with 2 and with -1 rounds to fp32 once more
    for n, got, base in (("dk", dk32, 2.0), ("dv", dv32, -1.0)):
        value, bound = want[n]
        ref.close(n, got, (value + base, bound + 2.0 ** -24 * (value.abs() + abs(base))))


def dev(*ts):
    return [t.to(DEV) for t in ts]


@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 64), (8, 2, 128), (16, 1, 128), (3, 3, 64),
                                        (12, 4, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 4), (700, 0), (100000, 1)])
def test_single_tokens(h_q, h_kv, d, window, sinks):
    """The newest token of each cached sequence.  Places longer than what a sequence holds:
    the rest of each is NaN and must not matter."""
    held = [1, 2, 63, 64, 65, 700, 1500, 129]
    room = [4, 2, 70, 64, 100, 701, 1600, 300]
    say(f"[single tokens] heads=({h_q},{h_kv}) d={d} window={window} sinks={sinks}")
    starts = np.cumsum([0] + room[:-1])
    tiles = tile_list([(int(s) + n - 1, int(s) + n, 0, h_q) for s, n in zip(starts, held)])
    n_kv = sum(room) + 5
    q, k, v, _ = tensors(d + window, len(held), n_kv, h_q, h_kv, d)
    ok = ref.visible(room, ref.positions(tiles), n_kv, window, sinks)
    want = ref.attention(q, k, v, ok, ref.coverage(tiles, len(held), h_q))
    empty = torch.ones(n_kv, dtype=torch.bool)
    for s, n in zip(starts, held):
        empty[int(s):int(s) + n] = False
    k[empty], v[empty] = torch.nan, torch.nan
    o, lse = pl.libra_attn_window_fwd(*dev(q, k, v), offsets(room),
                                      pl.tiles_to_device(tiles, DEV), window=window, sinks=sinks)
    torch.cuda.synchronize()
    ref.close("o", o, want["o"])
    ref.close("lse", lse, want["lse"])


@pytest.mark.parametrize("h_q,h_kv,d,window", [(4, 1, 64, 20000), (8, 2, 128, 9000),
                                               (2, 1, 128, 17001), (5, 1, 64, 2000)])
def test_single_tokens_of_long_caches(h_q, h_kv, d, window):
    """Two sequences whose keys are cut into many ranges, and one of two key blocks."""
    held, sinks = [17000, 70, 9990], 5
    say(f"[long caches] heads=({h_q},{h_kv}) d={d} window={window}")
    ends = np.cumsum(held)
    tiles = tile_list([(int(e) - 1, int(e), 0, h_q) for e in ends])
    n_kv = int(ends[-1])
    q, k, v, _ = tensors(d + window, len(held), n_kv, h_q, h_kv, d)
    ok = ref.visible(held, ref.positions(tiles), n_kv, window, sinks)
    want = ref.attention(q, k, v, ok, ref.coverage(tiles, len(held), h_q))
    o, lse = pl.libra_attn_window_fwd(*dev(q, k, v), offsets(held),
                                      pl.tiles_to_device(tiles, DEV), window=window, sinks=sinks)
    torch.cuda.synchronize()
    ref.close("o", o, want["o"])
    ref.close("lse", lse, want["lse"])


def test_single_tokens_of_head_shards_and_longer_tiles():
    """No more rows than tiles, but not one row to a tile: eight head shards of a 20-row and a
    150-row tile beside single rows, tiles out of range among them, which are counted."""
    h_q, h_kv, d, lengths = 8, 4, 64, [300, 40, 260]
    spans = [(100, 250, h, h + 1) for h in range(8)] + [(330, 350, h, h + 1) for h in range(8)]
    spans += [(299, 300, 0, 8), (339, 340, 0, 3), (598, 600, 0, 8)]
    tiles = tile_list(spans)
    rows = int((tiles["q_row"] + tiles["q_end"] - tiles["q_begin"]).max())
    bad = np.zeros(200, dtype=pl.TILE_DTYPE)
    bad["q_begin"], bad["q_end"], bad["head_end"] = 5, 5, 8         # empty
    bad[0] = (10, 11, rows, 0, 0, 8, 0, 0, 0, 0)                      # past the Q rows
    bad[1] = (10, 11, 0, 0, 0, 9, 0, 0, 0, 0)                         # past the heads
    say(f"[single tokens, odd tiles] rows={rows} tiles={len(tiles)}+{len(bad)}")
    every = np.concatenate([bad[:100], tiles, bad[100:]])
    assert rows <= len(every)
    n_kv = sum(lengths)
    q, k, v, _ = tensors(3, rows, n_kv, h_q, h_kv, d)
    cov = ref.coverage(tiles, rows, h_q)
    ok = ref.visible(lengths, ref.positions(tiles), n_kv, 70, 2)
    want = ref.attention(q, k, v, ok, cov)
    sizes = (len(every), len(lengths), rows, n_kv, h_q, h_kv, d)
    ws = pl.alloc_workspace(pl.libra_attn_window_workspace_size(*sizes, False, window=70, sinks=2),
                            DEV)
    qd = q.to(DEV)
    o, lse = torch.full_like(qd, 7.0), torch.full((h_q, rows), 7.0, device=DEV)
    pl.libra_attn_window_fwd(qd, *dev(k, v), offsets(lengths), pl.tiles_to_device(every, DEV),
                             window=70, sinks=2, o=o, lse=lse, workspace=ws)
    assert pl.libra_attn_skipped_tiles(ws) == len(bad)
    ref.close("o", o, want["o"], cov)
    ref.close("lse", lse, want["lse"], cov.T)
    assert (o.cpu()[~cov] == 7).all() and (lse.cpu()[~cov.T] == 7).all()


@pytest.mark.parametrize("rows_per_tile", [1, 40])
def test_many_sequences(rows_per_tile):
    """More samples than the preparation keeps in LDS, of one to 40 keys each."""
    rng = np.random.default_rng(5)
    lengths = rng.integers(1, 41, size=2600).tolist()
    h_q, h_kv, d, window = 4, 2, 64, 9
    ends = np.cumsum(lengths)
    if rows_per_tile == 1:
        tiles = tile_list([(int(e) - 1, int(e), 0, h_q) for e in ends])
    else:
        tiles = blocks(int(ends[-1]), rows_per_tile, h_q)
    say(f"[many sequences] {len(lengths)} samples, {len(tiles)} tiles")
    pos = ref.positions(tiles)
    n_q, n_kv = len(pos), sum(lengths)
    q, k, v, do = tensors(1, n_q, n_kv, h_q, h_kv, d)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    qd, kd, vd, dod = dev(q, k, v, do)
    o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, window=window, sinks=2)
    dq, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, window=window, sinks=2)
    torch.cuda.synchronize()
    # samples one by one would take long: the first, a middle and the last 60
    for a in (0, 1300, 2540):
        b = a + 60
        k0, k1 = int(ends[a] - lengths[a]), int(ends[b - 1])
        r = torch.nonzero((pos >= k0) & (pos < k1))[:, 0]
        ok = ref.visible(lengths[a:b], pos[r] - k0, k1 - k0, window, 2)
        cov = torch.ones((len(r), h_q), dtype=torch.bool)
        want = ref.attention(q[r], k[k0:k1], v[k0:k1], ok, cov, dout=do[r])
        ref.close("o", o[r], want["o"])
        ref.close("lse", lse[:, r], want["lse"])
        ref.close("dq", dq[r], want["dq"])
        ref.close("dk", dk[k0:k1], want["dk"])
        ref.close("dv", dv[k0:k1], want["dv"])


@pytest.mark.parametrize("h_q,h_kv,d,lengths,B,window,sinks", [
    (32, 4, 128, [900, 2700, 55, 1, 700], 512, 600, 4),
    (32, 8, 64, [4000, 300], 1237, 1111, 40),
    (4, 1, 64, [34000], 34000, 300, 0),
])
def test_larger_calls(h_q, h_kv, d, lengths, B, window, sinks):
    """Lists that many workgroups build; whole gradients against float64 on the GPU."""
    say(f"[window larger] lengths={lengths} heads=({h_q},{h_kv}) d={d} window={window}")
    n = sum(lengths)
    tiles = blocks(n, B, h_q)
    pos = ref.positions(tiles)
    qd, kd, vd, dod = dev(*tensors(n, n, n, h_q, h_kv, d))
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    mask = dict(window=window, sinks=sinks)
    o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
    dq, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask)
    torch.cuda.synchronize()
    if n > 10000:   # a stretch of rows, and the keys that only it reaches
        a, b = 20000, 23000
        keys = slice(a - window + 1, b)
        ok = ref.visible([b], pos[a:b], b, window, 0)[:, keys]
        want = ref.attention(qd[a:b], kd[keys], vd[keys], ok,
                             torch.ones((b - a, h_q), dtype=torch.bool), dout=dod[a:b])
        ref.close("o", o[a:b], want["o"])
        ref.close("dq", dq[a:b], want["dq"])
        inner = slice(window - 1, b - a)   # of `keys`, those from row a to b - window
        for name, got in (("dk", dk), ("dv", dv)):
            ref.close(name, got[a:b - window + 1],
                      tuple(x[inner][:b - window + 1 - a] for x in want[name]))
        return
    ok = ref.visible(lengths, pos, n, window, sinks)
    want = ref.attention(qd, kd, vd, ok, torch.ones((n, h_q), dtype=torch.bool), dout=dod)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.close(name, got, want[name])


def test_what_lies_outside_does_not_matter():
    """NaN in rows that no tile covers, in keys past the last covered row, in samples that no
    tile touches and behind the last sample."""
    h_q, h_kv, d, lengths, window, sinks = 4, 2, 128, [400, 900, 200], 100, 3
    tiles = tile_list([(500, 700, 0, 2), (650, 800, 2, 4), (850, 860, 1, 3)])
    pos = ref.positions(tiles)
    n_q, n_kv = len(pos) + 7, sum(lengths) + 9
    say("[window, NaN outside]")
    q, k, v, do = tensors(8, n_q, n_kv, h_q, h_kv, d)
    cov = torch.cat([ref.coverage(tiles, len(pos), h_q), torch.zeros((7, h_q), dtype=torch.bool)])
    ok = ref.visible(lengths, torch.cat([pos, torch.full((7,), -1)]), n_kv, window, sinks)
    want = ref.attention(q, k, v, ok, cov, dout=do)
    q[~cov], do[~cov] = torch.nan, torch.nan
    seen = torch.zeros(n_kv, dtype=torch.bool)
    seen[400:860] = True
    k[~seen], v[~seen] = torch.nan, torch.nan
    qd, kd, vd, dod = dev(q, k, v, do)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    mask = dict(window=window, sinks=sinks)
    o, lse = torch.full_like(qd, torch.nan), torch.full((h_q, n_q), torch.nan, device=DEV)
    pl.libra_attn_window_fwd(qd, kd, vd, cu, td, o=o, lse=lse, **mask)
    dq, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask)
    held = [pl.libra_ckpt8_pack(x) for x in (qd, kd, vd, o)]
    dq8, dk8, dv8 = pl.libra_attn_bwd_ckpt8(*held, lse, dod, cu, td, **mask)
    torch.cuda.synchronize()
    ref.close("o", o, want["o"], cov)
    ref.close("lse", lse, want["lse"], cov.T)
    ref.close("dq", dq, want["dq"], cov)
    for name, got in (("dk", dk), ("dv", dv)):
        ref.close(name, got, want[name])
    assert torch.isfinite(dq8.cpu()[cov]).all()
    assert torch.isfinite(dk8).all() and torch.isfinite(dv8).all()
    untouched = torch.ones(n_kv, dtype=torch.bool)
    untouched[400:860] = False
    assert (dk8.cpu()[untouched] == 0).all() and (dv8.cpu()[untouched] == 0).all()


@pytest.mark.parametrize("h_q,h_kv,d,rows,window,sinks", [
    (8, 2, 128, 1, 100, 4), (8, 2, 64, 1, 1, 0), (16, 2, 128, 1, 700, 70), (3, 3, 64, 1, 65, 0),
    (4, 1, 128, 20, 90, 3), (2, 1, 64, 61, 64, 130), (4, 4, 128, 128, 1, 1)])
def test_keys_given_up(h_q, h_kv, d, rows, window, sinks):
    """The newest rows of cached sequences whose keys between the sinks and the window of the
    first of those rows are NaN or infinite, as are those past the last row.  At most 128 rows
    times heads of a KV group, so that a tile's rows are one work item."""
    held, room = [rows, 129, 1000, 1337, 650], [rows + 3, 200, 1000, 1500, 651]
    say(f"[keys given up] heads=({h_q},{h_kv}) d={d} rows={rows} window={window} sinks={sinks}")
    starts = np.cumsum([0] + room[:-1])
    tiles = tile_list([(int(s) + n - rows, int(s) + n, 0, h_q) for s, n in zip(starts, held)])
    n_q, n_kv = rows * len(held), sum(room)
    q, k, v, _ = tensors(rows + window, n_q, n_kv, h_q, h_kv, d)
    ok = ref.visible(room, ref.positions(tiles), n_kv, window, sinks)
    want = ref.attention(q, k, v, ok, ref.coverage(tiles, n_q, h_q))
    junk = ~ok.any(0)
    assert junk.sum() > 100
    k[junk], v[junk] = torch.nan, torch.inf
    o, lse = pl.libra_attn_window_fwd(*dev(q, k, v), offsets(room),
                                      pl.tiles_to_device(tiles, DEV), window=window, sinks=sinks)
    torch.cuda.synchronize()
    ref.close("o", o, want["o"])
    ref.close("lse", lse, want["lse"])


def _step(q, k, v, do, cu, td, mask, bufs):
    """Forward, checkpoint and both backwards into `bufs`, as one layer runs them."""
    o, lse, dq, dk, dv, ws, held, dq8, dk8, dv8 = bufs
    pl.libra_attn_window_fwd(q, k, v, cu, td, o=o, lse=lse, workspace=ws, **mask)
    for x, (n, e) in zip((q, k, v, o), held):
        pl.libra_ckpt8_pack(x, q=n, e=e)
    pl.libra_attn_window_bwd(q, k, v, o, lse, do, cu, td, dq=dq, dk=dk, dv=dv, workspace=ws,
                             **mask)
    pl.libra_attn_bwd_ckpt8(*held, lse, do, cu, td, dq=dq8, dk=dk8, dv=dv8, workspace=ws, **mask)


def _buffers(q, k, T, n, mask):
    sizes = (T, n, q.shape[0], k.shape[0], q.shape[1], k.shape[1], q.shape[2])
    need = max(pl.libra_attn_window_workspace_size(*sizes, False, **mask),
               pl.libra_attn_window_workspace_size(*sizes, True, **mask),
               pl.libra_attn_bwd_ckpt8_workspace_size(*sizes, **mask))
    held = [(torch.zeros(x.shape, dtype=torch.int8, device=DEV),
             torch.zeros((*x.shape[:-1], x.shape[-1] // 32), dtype=torch.uint8, device=DEV))
            for x in (q, k, k, q)]
    z = torch.zeros_like
    return (z(q), torch.zeros((q.shape[1], q.shape[0]), device=DEV), z(q), z(k), z(k),
            torch.full((need,), 0xff, dtype=torch.uint8, device=DEV), held, z(q), z(k), z(k))


def _results(bufs):
    o, lse, dq, dk, dv, _, held, dq8, dk8, dv8 = bufs
    return [x.clone() for x in (o, lse, dq, dk, dv, *(t for p in held for t in p), dq8, dk8, dv8)]


@pytest.mark.parametrize("case", ["small", "large"])
def test_repeats_streams_and_graphs(case):
    """The same bits from one call to the next, on another stream than the tensors', and from
    two captured graphs with workspaces of their own whose replays alternate with eager work
    (dirty workspaces throughout)."""
    h_q, h_kv, d, lengths, B = {"small": (4, 2, 64, [900, 30], 200),
                                "large": (32, 8, 128, [3500, 700, 31], 1024)}[case]
    mask = dict(window=200, sinks=5)
    n = sum(lengths)
    say(f"[graphs {case}] lengths={lengths}")
    tiles = blocks(n, B, h_q)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    sets = [dev(*tensors(s, n, n, h_q, h_kv, d)) for s in (1, 2)]
    bufs = [_buffers(*t[:2], len(tiles), len(lengths), mask) for t in sets]
    want = []
    for t, b in zip(sets, bufs):
        _step(*t, cu, td, mask, b)
        want.append(_results(b))
        _step(*t, cu, td, mask, b)
        assert all(torch.equal(x, y) for x, y in zip(want[-1], _results(b)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(*sets[0], cu, td, mask, bufs[0])
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want[0], _results(bufs[0])))
    graphs = []
    for t, b in zip(sets, bufs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _step(*t, cu, td, mask, b)
        graphs.append(g)
    for turn in range(4):
        for g, b, w in zip(graphs, bufs, want):
            for x in _results_in(b):
                x.zero_()
            g.replay()
            eager = sets[0][0].float().sum()   # the program's own work in between
            assert torch.isfinite(eager)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(w, _results(b))), f"replay {turn}"


def _results_in(bufs):
    o, lse, dq, dk, dv, _, held, dq8, dk8, dv8 = bufs
    return [o, lse, dq, dk, dv, *(t for p in held for t in p), dq8, dk8, dv8]


def test_two_calls_at_once():
    """Layers on two streams with workspaces of their own, posted without waiting."""
    h_q, h_kv, d, lengths, mask = 16, 4, 128, [2500, 900, 64], dict(window=300, sinks=3)
    n = sum(lengths)
    say(f"[two at once] lengths={lengths}")
    tiles = blocks(n, 512, h_q, 2)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    sets = [dev(*tensors(s, n, n, h_q, h_kv, d)) for s in (3, 4)]
    bufs = [_buffers(*t[:2], len(tiles), len(lengths), mask) for t in sets]
    want = []
    for t, b in zip(sets, bufs):
        _step(*t, cu, td, mask, b)
        want.append(_results(b))
        for x in _results_in(b):
            x.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        for st, t, b in zip(streams, sets, bufs):
            with torch.cuda.stream(st):
                _step(*t, cu, td, mask, b)
    torch.cuda.synchronize()
    for b, w in zip(bufs, want):
        assert all(torch.equal(x, y) for x, y in zip(w, _results(b)))


def test_last_sample_past_the_keys():
    """Offsets of a sample that goes on behind the last row of K and V: as if it ended there."""
    h_q, h_kv, d, n, mask = 4, 2, 64, 1200, dict(window=900, sinks=4)
    say("[window, last sample past the keys]")
    tiles = blocks(n, 256, h_q)
    q, k, v, do = tensors(9, n, n, h_q, h_kv, d)
    cu = torch.tensor([0, 200, 50000], device=DEV)
    qd, kd, vd, dod = dev(q, k, v, do)
    td = pl.tiles_to_device(tiles, DEV)
    want = ref.attention(q, k, v, ref.visible([200, 1000], ref.positions(tiles), n, 900, 4),
                         torch.ones((n, h_q), dtype=torch.bool), dout=do)
    o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
    got = (o, lse, *pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask))
    torch.cuda.synchronize()
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), got):
        ref.close(name, x, want[name])


def test_wide_window_is_causal():
    """A window of the longest sample: causal attention, within both calls' bounds."""
    h_q, h_kv, d, lengths = 8, 2, 128, [700, 64, 300]
    n = sum(lengths)
    say("[window = longest sample]")
    tiles = blocks(n, 256, h_q, 2)
    qd, kd, vd, dod = dev(*tensors(4, n, n, h_q, h_kv, d))
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    want = ref.attention(qd, kd, vd, ref.visible(lengths, ref.positions(tiles), n, 0, 0),
                         torch.ones((n, h_q), dtype=torch.bool), dout=dod)
    o, lse = pl.libra_attn_fwd(qd, kd, vd, cu, td)
    a = (o, lse, *pl.libra_attn_bwd(qd, kd, vd, o, lse, dod, cu, td))
    ow, lw = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, window=700)
    b = (ow, lw, *pl.libra_attn_window_bwd(qd, kd, vd, ow, lw, dod, cu, td, window=700))
    for name, x, y in zip(("o", "lse", "dq", "dk", "dv"), a, b):
        ref.close(name, x, want[name])
        ref.close(name, y, want[name])


def test_cache_past_32_bit_offsets():
    """K and V of more than 2^31 elements: rows at both ends of a long cache."""
    h_q, h_kv, d = 8, 8, 128
    n_kv = (1 << 31) // (h_kv * d) + 5000
    say(f"[window] {n_kv} keys")
    window, sinks = 300, 2
    tiles = tile_list([(n_kv - 1, n_kv, 0, h_q), (n_kv - 200, n_kv - 100, 0, h_q), (7, 9, 0, h_q)])
    pos = ref.positions(tiles)
    n_q = len(pos)
    keys = torch.cat([torch.arange(0, 16), torch.arange(n_kv - 600, n_kv)])
    q, ks, vs, do = tensors(6, n_q, len(keys), h_q, h_kv, d)
    kd = torch.zeros((n_kv, h_kv, d), dtype=torch.bfloat16, device=DEV)
    vd = torch.zeros_like(kd)
    at = keys.to(DEV)
    kd[at], vd[at] = ks.to(DEV), vs.to(DEV)
    p, kk = pos[:, None], keys[None, :]
    ok = (kk <= p) & ((kk > p - window) | (kk < sinks))
    want = ref.attention(q, ks, vs, ok, torch.ones((n_q, h_q), dtype=torch.bool), dout=do)
    qd, dod = dev(q, do)
    cu = offsets([n_kv])
    mask = dict(window=window, sinks=sinks)
    one = pl.tiles_to_device(tiles[:1], DEV)   # a single token
    o1, _ = pl.libra_attn_window_fwd(qd[:1].contiguous(), kd, vd, cu, one, **mask)
    ref.close("o", o1, tuple(x[:1] for x in want["o"]))
    td = pl.tiles_to_device(tiles, DEV)
    o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
    dq, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask)
    torch.cuda.synchronize()
    ref.close("o", o, want["o"])
    ref.close("dq", dq, want["dq"])
    ref.close("dk", dk[at], want["dk"])
    ref.close("dv", dv[at], want["dv"])
    assert not bool(dk[16:n_kv - 600].any()) and not bool(dv[16:n_kv - 600].any())


def test_softmax_scale_and_large_scores():
    """A scale of the caller's, and scores of some hundreds (rows in which one key counts)."""
    h_q, h_kv, d, lengths = 4, 2, 64, [500]
    say("[window, large scores]")
    tiles = blocks(500, 128, h_q)
    q, k, v, do = tensors(2, 500, 500, h_q, h_kv, d, size=4.0)
    qd, kd, vd, dod = dev(q, k, v, do)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    mask = dict(window=90, sinks=2, softmax_scale=0.5)
    ok = ref.visible(lengths, ref.positions(tiles), 500, 90, 2)
    want = ref.attention(q, k, v, ok, torch.ones((500, h_q), dtype=torch.bool), scale=0.5)
    o, lse = pl.libra_attn_window_fwd(qd, kd, vd, cu, td, **mask)
    dq, dk, dv = pl.libra_attn_window_bwd(qd, kd, vd, o, lse, dod, cu, td, **mask)
    torch.cuda.synchronize()
    # scores reach 0.5 * 64 * 16 and more: their fp32 sums are off by up to 64 roundings of
    # terms that sum to some 1000, 64 * 2^-24 * 1000 = 4e-3 at most, relative in P
    far = 64 * 2.0 ** -24 * float((q.double().abs().amax() * k.double().abs().sum(-1).amax()) * 0.5)
    value, bound = want["o"]
    weight = ref.attention(q, k, v.abs(), ok, torch.ones((500, h_q), dtype=torch.bool),
                           scale=0.5)["o"][0]
    ref.close("o", o, (value, bound + 2 * far * weight))
    ref.close("lse", lse, (want["lse"][0], want["lse"][1] + far))
    for x in (dq, dk, dv):
        assert torch.isfinite(x).all()
