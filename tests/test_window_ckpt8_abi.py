"""Refusals of the windowed attention and 8-bit checkpoint entry points: all on the host,
before anything is enqueued."""
import ctypes as C

import pytest
import torch

import paper_2607_23250_amd as pl

FAKE = C.c_void_p(4096)


def size(window, sinks, backward=False, d=64, h=(4, 2), rows=1000):
    return pl.libra_attn_window_workspace_size(8, 2, rows, rows, *h, d, backward, window=window,
                                               sinks=sinks)


def test_workspace_sizes():
    assert size(100, 4) > 0 and size(100, 4, True) > size(100, 4)
    assert size(1 << 40, 1024, True) > 0            # past the rows: as the rows
    for bad in (dict(window=0, sinks=0), dict(window=-1, sinks=0), dict(window=5, sinks=-1),
                dict(window=5, sinks=1025), dict(window=5, sinks=0, d=96),
                dict(window=5, sinks=0, h=(4, 3))):
        assert size(**bad) == 0 and size(**bad, backward=True) == 0
    held = pl.libra_attn_bwd_ckpt8_workspace_size
    assert held(8, 2, 1000, 1000, 4, 2, 64) > pl.libra_attn_workspace_size(8, 2, 1000, 1000, 4, 2,
                                                                           64, True)
    assert held(8, 2, 1000, 1000, 4, 2, 64, window=10, sinks=3) > 0
    assert held(8, 2, 1000, 1000, 4, 2, 64, sinks=3) == 0       # sinks without a window
    assert held(8, 2, 1000, 1000, 4, 2, 64, window=-3) == 0
    # far sinks take space only where samples can be long enough
    assert size(900, 64, True) == size(900, 0, True)
    assert size(100, 64, True) > size(100, 0, True)


def fwd(window=5, sinks=0, d=64, tiles=1, ptr=FAKE, ws=FAKE, ws_bytes=1 << 40, h_kv=2):
    return pl.lib().libra_attn_window_fwd(ptr, ptr, ptr, ptr, 1, ptr, tiles, 10, 10, 4, h_kv, d,
                                          window, sinks, 0.0, ptr, ptr, ws, ws_bytes, None)


def bwd(window=5, sinks=0, d=64, tiles=1, ptr=FAKE, ws=FAKE, ws_bytes=1 << 40, flags=0, dk=FAKE):
    return pl.lib().libra_attn_window_bwd(ptr, ptr, ptr, ptr, ptr, ptr, ptr, 1, ptr, tiles, 10, 10,
                                          4, 2, d, window, sinks, 0.0, ptr, dk, dk, flags, ws,
                                          ws_bytes, None)


def bwd8(window=5, sinks=0, d=64, tiles=1, ptr=FAKE, ws=FAKE, ws_bytes=1 << 40, flags=0,
         held=(4096, 4096)):
    c = C.byref(pl._Ckpt8(*held))
    return pl.lib().libra_attn_bwd_ckpt8(c, c, c, c, ptr, ptr, ptr, 1, ptr, tiles, 10, 10, 4, 2, d,
                                         window, sinks, 0.0, ptr, FAKE, FAKE, flags, ws, ws_bytes,
                                         None)


@pytest.mark.parametrize("call", [fwd, bwd, bwd8])
def test_attention_refusals(call):
    assert call(window=-1) == pl.LIBRA_EINVAL
    assert call(sinks=-1) == pl.LIBRA_EINVAL
    assert call(sinks=1025) == pl.LIBRA_EUNSUPPORTED
    assert b"1025" in pl.lib().libra_last_error()
    assert call(d=96) == pl.LIBRA_EUNSUPPORTED
    assert call(tiles=-1) == pl.LIBRA_EINVAL
    assert call(ptr=None) == pl.LIBRA_EINVAL
    assert call(ws=None) == pl.LIBRA_EINVAL
    assert call(ws=C.c_void_p(4096 + 16)) == pl.LIBRA_EINVAL
    assert call(ws_bytes=100) == pl.LIBRA_ENOSPC


def test_attention_refusals_of_one_direction():
    assert fwd(window=0) == pl.LIBRA_EINVAL and bwd(window=0) == pl.LIBRA_EINVAL
    assert bwd8(window=0, sinks=2) == pl.LIBRA_EINVAL     # a causal call has no sinks
    assert fwd(tiles=0, ptr=None, ws=None) == pl.LIBRA_OK   # nothing to do
    assert fwd(h_kv=3) == pl.LIBRA_EINVAL
    assert bwd(flags=2) == pl.LIBRA_EINVAL and bwd8(flags=2) == pl.LIBRA_EINVAL
    assert bwd(dk=None) == pl.LIBRA_EINVAL
    assert bwd8(held=(None, 4096)) == pl.LIBRA_EINVAL
    assert bwd8(held=(4096, None)) == pl.LIBRA_EINVAL
    assert bwd8(held=(4097, 4096)) == pl.LIBRA_EINVAL


@pytest.mark.parametrize("call", ["fwd", "bwd", "bwd8"])
def test_misaligned_pointers(call):
    """Each pointer in turn off by less than its alignment."""
    L, c = pl.lib(), C.byref(pl._Ckpt8(4096, 4096))
    names = {"fwd": "q k v cu tiles o lse".split(), "bwd8": "lse do cu tiles dq dk dv".split(),
             "bwd": "q k v o lse do cu tiles dq dk dv".split()}[call]
    for bad in names:
        off = {"lse": 2, "cu": 4, "tiles": 4}.get(bad, 8)
        p = {n: C.c_void_p(4096 + (off if n == bad else 0)) for n in names}
        if call == "fwd":
            rc = L.libra_attn_window_fwd(p["q"], p["k"], p["v"], p["cu"], 1, p["tiles"], 1, 10, 10,
                                         4, 2, 64, 5, 0, 0.0, p["o"], p["lse"], FAKE, 1 << 40, None)
        elif call == "bwd":
            rc = L.libra_attn_window_bwd(p["q"], p["k"], p["v"], p["o"], p["lse"], p["do"], p["cu"],
                                         1, p["tiles"], 1, 10, 10, 4, 2, 64, 5, 0, 0.0, p["dq"],
                                         p["dk"], p["dv"], 0, FAKE, 1 << 40, None)
        else:
            rc = L.libra_attn_bwd_ckpt8(c, c, c, c, p["lse"], p["do"], p["cu"], 1, p["tiles"], 1,
                                        10, 10, 4, 2, 64, 5, 0, 0.0, p["dq"], p["dk"], p["dv"], 0,
                                        FAKE, 1 << 40, None)
        assert rc == pl.LIBRA_EINVAL and b"aligned" in L.libra_last_error(), bad


@pytest.mark.parametrize("name", ["pack", "unpack"])
def test_ckpt8_refusals(name):
    def call(dtype=0, rows=4, cols=64, ld=64, x=FAKE, q=FAKE, e=FAKE):
        L = pl.lib()
        if name == "pack":
            return L.libra_ckpt8_pack(x, dtype, rows, cols, ld, q, e, None)
        return L.libra_ckpt8_unpack(q, e, rows, cols, dtype, ld, x, None)
    assert call(dtype=2) == pl.LIBRA_EUNSUPPORTED and call(dtype=-1) == pl.LIBRA_EUNSUPPORTED
    assert call(rows=-1) == pl.LIBRA_EINVAL
    assert call(cols=63) == pl.LIBRA_EINVAL and call(cols=-32) == pl.LIBRA_EINVAL
    assert call(ld=63) == pl.LIBRA_EINVAL                       # rows overlap
    assert call(ld=68) == pl.LIBRA_EINVAL                       # not 16 bytes
    assert call(dtype=1, ld=66) == pl.LIBRA_EINVAL
    assert call(x=None) == pl.LIBRA_EINVAL and call(q=None) == pl.LIBRA_EINVAL
    assert call(e=None) == pl.LIBRA_EINVAL
    assert call(x=C.c_void_p(4104)) == pl.LIBRA_EINVAL
    assert call(q=C.c_void_p(4104)) == pl.LIBRA_EINVAL
    assert call(rows=1 << 60, ld=1 << 20, cols=1 << 20) == pl.LIBRA_EOVERFLOW
    assert call(rows=0, x=None, q=None, e=None) == pl.LIBRA_OK
    assert call(cols=0, ld=0, x=None, q=None, e=None) == pl.LIBRA_OK


def test_binding_refuses_what_it_cannot_pass_on():
    b16 = torch.bfloat16
    x = torch.zeros((4, 2, 64), dtype=b16)
    cu = torch.tensor([0, 4])
    tiles = torch.zeros(56, dtype=torch.uint8)
    with pytest.raises(ValueError):   # host tensors
        pl.libra_ckpt8_pack(x)
    with pytest.raises(ValueError):
        pl.libra_ckpt8_unpack(x.to(torch.int8), torch.zeros((4, 2, 2), dtype=torch.uint8))
    with pytest.raises(ValueError):
        pl.libra_attn_window_fwd(x, x, x, cu, tiles, window=3)
    with pytest.raises(ValueError):
        pl.libra_attn_window_bwd(x, x, x, x, torch.zeros((2, 4)), x, cu, tiles, window=3)
    held = (x.to(torch.int8), torch.zeros((4, 2, 2), dtype=torch.uint8))
    with pytest.raises(ValueError):
        pl.libra_attn_bwd_ckpt8(held, held, held, held, torch.zeros((2, 4)), x, cu, tiles)
    assert pl._rows_cols_ld(torch.zeros((5, 3, 64)), "x") == (15, 64, 64)
    assert pl._rows_cols_ld(torch.zeros((5, 200))[:, 32:96], "x") == (5, 64, 200)
    assert pl._rows_cols_ld(torch.zeros((5, 4, 64))[:, :1], "x") == (5, 64, 256)
    assert pl._rows_cols_ld(torch.zeros((5, 4, 64))[:1, 1:2], "x") == (1, 64, 64)
    for bad in (torch.zeros((5, 4, 64))[:, 1:3], torch.zeros((64, 5)).T):
        with pytest.raises(ValueError):
            pl._rows_cols_ld(bad, "x")
