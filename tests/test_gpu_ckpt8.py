"""GPU tests of the 8-bit activation checkpoints: libra_ckpt8_pack / libra_ckpt8_unpack to
the bit against their definition in float64, and libra_attn_bwd_ckpt8 against dense
attention gradients in float64 (bounds: window_ref.py) and, to the bit, against itself on
held values that were packed twice."""
import numpy as np
import pytest
import torch

import paper_2607_23250_amd as pl
import window_ref as ref
from gpu_util import DEV, say
from test_gpu_window import blocks, offsets, tensors, tile_list

pytestmark = pytest.mark.gpu


def held(x):
    """(integers, exponent bytes, values) of x by the definition, in float64."""
    g = x.double().reshape(-1, 32)
    top = g.abs().amax(1, keepdim=True)
    bad = ~torch.isfinite(top)
    e = torch.full(top.shape, -126.0, dtype=torch.float64)
    for _ in range(260):   # the smallest unit that fits, one doubling at a time
        e = torch.where(~bad & (e < 121) & (torch.round(top * torch.exp2(-e)) > 127), e + 1, e)
    n = torch.where(bad, 0.0, torch.round(g * torch.exp2(-e)).clamp(-127, 127))
    value = torch.where(bad, torch.nan, n * torch.exp2(e))
    byte = torch.where(bad, 255.0, e + 127)
    return (n.reshape(x.shape).to(torch.int8), byte.reshape(*x.shape[:-1], -1).to(torch.uint8),
            value.reshape(x.shape))


def same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def check_pack(x, x_dev=None):
    x_dev = x.to(DEV) if x_dev is None else x_dev
    q, e = pl.libra_ckpt8_pack(x_dev)
    n, byte, value = held(x)
    assert torch.equal(q.cpu(), n) and torch.equal(e.cpu(), byte)
    for dtype in (torch.bfloat16, torch.float32):
        y = pl.libra_ckpt8_unpack(q, e, dtype=dtype)
        assert y.dtype == dtype and same(y.cpu().double(), value)   # held values are exact
        q2, e2 = pl.libra_ckpt8_pack(y)
        z = pl.libra_ckpt8_unpack(q2, e2, dtype=torch.float32)
        assert same(z.cpu().double(), value)                        # and held again


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1, 32), (3, 64), (7, 5, 96), (1000, 32), (129, 8, 128),
                                   (2, 3, 5, 64)])
def test_pack_unpack(dtype, shape):
    say(f"[ckpt8] {dtype} {shape}")
    gen = torch.Generator().manual_seed(sum(shape))
    x = torch.randn(shape, generator=gen) * torch.exp(3 * torch.randn(shape, generator=gen))
    check_pack(x.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pack_of_extreme_values(dtype):
    say(f"[ckpt8 extremes] {dtype}")
    info = torch.finfo(dtype)
    tiny = float(torch.tensor(2.0 ** (-133 if dtype == torch.bfloat16 else -149)))
    groups = [[0.0], [-0.0], [info.max, -info.max, 1.0], [info.tiny], [tiny, -tiny], [tiny * 3],
              [127.0, 126.5, -127.0, 0.5, 1.5], [127.5, 1.0], [127.25, 63.5], [128.0], [-127.5],
              [255.0, 254.0], [np.inf, 1.0], [-np.inf], [np.nan, 2.0], [2.0 ** -120, 2.0 ** -127],
              [2.0 ** -119 * 1.9921875], [info.max], [1.0, 2.0 ** -7, 2.0 ** -8]]
    x = torch.zeros((len(groups), 32))
    for i, g in enumerate(groups):
        x[i, :len(g)] = torch.tensor(g)
        x[i, 31] = g[0]
    check_pack(x.to(dtype))


def test_pack_of_every_bf16_value():
    """Each value alone with zeros, and beside a power of two that sets the unit."""
    say("[ckpt8 every bf16]")
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros((65536, 32), dtype=torch.bfloat16)
    x[:, 5] = bits
    x[:, 20] = bits * 0.375
    check_pack(x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pack_and_unpack_of_strided_rows(dtype):
    """q, k and v as slices of one fused projection's output, and unpacked into such slices."""
    say(f"[ckpt8 strided] {dtype}")
    gen = torch.Generator().manual_seed(5)
    wide = torch.randn((37, 4 * 64 + 96), generator=gen).to(dtype)
    wd = wide.to(DEV)
    for a, b in ((0, 256), (256, 352), (64, 128)):
        check_pack(wide[:, a:b].contiguous(), wd[:, a:b])
    heads = wd[:, :256].view(37, 4, 64)[:, 1:3]   # two axes that do not lie at one stride
    with pytest.raises(ValueError):
        pl.libra_ckpt8_pack(heads)
    q, e = pl.libra_ckpt8_pack(wd[:, 64:128])
    out = torch.full((37, 352), 3.0, dtype=dtype, device=DEV)
    pl.libra_ckpt8_unpack(q, e, out=out[:, 256:320])
    assert torch.equal(out[:, 256:320].cpu().double(), held(wide[:, 64:128].contiguous())[2])
    assert (out[:, :256] == 3).all() and (out[:, 320:] == 3).all()


def test_pack_past_32_bit_offsets():
    """Elements past 2^31: the last rows of a large tensor."""
    rows, cols = (1 << 31) // 4096 + 3, 4096
    say(f"[ckpt8] {rows} x {cols}")
    x = torch.ones((rows, cols), dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator().manual_seed(9)
    tail = torch.randn((3, cols), generator=gen).to(torch.bfloat16)
    x[-3:] = tail.to(DEV)
    q, e = pl.libra_ckpt8_pack(x)
    n, byte, value = held(tail)
    assert torch.equal(q[-3:].cpu(), n) and torch.equal(e[-3:].cpu(), byte)
    assert bool((q[:-3] == 64).all()) and bool((e[:-3] == 121).all())
    y = pl.libra_ckpt8_unpack(q, e)
    assert torch.equal(y[-3:].cpu().double(), value) and bool((y[:-3] == 1).all())


def test_empty():
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device=DEV)
    q, e = pl.libra_ckpt8_pack(x)
    assert q.shape == (0, 64) and e.shape == (0, 2)
    assert pl.libra_ckpt8_unpack(q, e).shape == (0, 64)


CASES = {   # lengths, tiles, heads, d, window, sinks
    "causal": ([500, 3, 97], blocks(600, 128, 4), (4, 2), 128, 0, 0),
    "causal_d64": ([900], blocks(900, 256, 6, 2), (6, 2), 64, 0, 0),
    "window": ([700, 200], blocks(900, 256, 4), (4, 1), 128, 100, 0),
    "far_sinks": ([1200], blocks(1200, 256, 4, 2), (4, 2), 64, 130, 5),
    "part": ([800], tile_list([(300, 431, 0, 2), (700, 800, 1, 3)]), (4, 2), 64, 90, 2),
    "odd": ([333], blocks(333, 100, 3), (3, 1), 128, 64, 1),
}


@pytest.mark.parametrize("name", CASES)
def test_backward_from_checkpoints(name):
    lengths, tiles, (h_q, h_kv), d, window, sinks = CASES[name]
    say(f"[bwd ckpt8 {name}] lengths={lengths} heads=({h_q},{h_kv}) d={d} window={window} "
        f"sinks={sinks}")
    pos = ref.positions(tiles)
    n_q, n_kv = len(pos), sum(lengths)
    q, k, v, do = tensors(len(name), n_q, n_kv, h_q, h_kv, d)
    cov = ref.coverage(tiles, n_q, h_q)
    ok = ref.visible(lengths, pos, n_kv, window, sinks)
    cu, td = offsets(lengths), pl.tiles_to_device(tiles, DEV)
    qd, kd, vd, dod = (t.to(DEV) for t in (q, k, v, do))
    o, lse = torch.zeros_like(qd), torch.zeros((h_q, n_q), device=DEV)
    # the layer as it runs: forward, checkpoint, backward
    if window:
        pl.libra_attn_window_fwd(qd, kd, vd, cu, td, o=o, lse=lse, window=window, sinks=sinks)
    else:
        pl.libra_attn_fwd(qd, kd, vd, cu, td, o=o, lse=lse)
    packs = [pl.libra_ckpt8_pack(x) for x in (qd, kd, vd, o)]
    dq = torch.full_like(qd, 7.0)
    _, dk, dv = pl.libra_attn_bwd_ckpt8(*packs, lse, dod, cu, td, window=window, sinks=sinks,
                                        dq=dq)
    torch.cuda.synchronize()
    qh, kh, vh, oh = (held(x.cpu())[2] for x in (qd, kd, vd, o))
    want = ref.attention(qh, kh, vh, ok, cov, dout=do, held=(oh, lse.cpu()))
    live = cov & ok.any(1)[:, None]
    ref.close("dq", dq, want["dq"], live)
    assert (dq.cpu()[~live] == 7).all()
    ref.close("dk", dk, want["dk"])
    ref.close("dv", dv, want["dv"])
    # fp32 sums, from two halves of the tiles
    dk2, dv2 = (torch.zeros(kd.shape, device=DEV) for _ in range(2))
    for part in (tiles[::2], tiles[1::2]):
        pl.libra_attn_bwd_ckpt8(*packs, lse, dod, cu, pl.tiles_to_device(part, DEV),
                                window=window, sinks=sinks, dk=dk2, dv=dv2, accumulate=True)
    torch.cuda.synchronize()
    ref.close("dk", dk2, (want["dk"][0], want["dk"][1] + 2.0 ** -23 * want["dk"][0].abs()))
    ref.close("dv", dv2, (want["dv"][0], want["dv"][1] + 2.0 ** -23 * want["dv"][0].abs()))
