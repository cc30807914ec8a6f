"""How large the workspaces of windowed calls get (host only)."""
import pytest

import paper_2607_23250_amd as pl


def backward(n, keys, h_kv, d, window, sinks):
    return pl.libra_attn_window_workspace_size(n, n, keys, keys, 2 * h_kv, h_kv, d, True,
                                               window=window, sinks=sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,keys,h_kv", [(1, 5000, 1), (40, 5000, 8), (400, 262144, 8),
                                         (5000, 1 << 20, 4), (1 << 20, 1 << 20, 64)])
@pytest.mark.parametrize("window", [1, 7, 128, 1000, 5000])
@pytest.mark.parametrize("sinks", [1, 32, 300, 1024])
def test_far_rows_of_sinks(d, n, keys, h_kv, window, sinks):
    """The partial sums over far rows take no more than the fp16 copies of K and V do, or 4096
    slots of 32 keys: whatever the samples are."""
    more = backward(n, keys, h_kv, d, window, sinks) - backward(n, keys, h_kv, d, window, 0)
    slots = max(keys * h_kv // 64, 4096)
    # 256 slots beyond those; an item of 32 bytes and a record of 8 each, a list, alignment
    assert 0 <= more <= (slots + 256) * (64 * d * 4 + 40) + 4 * keys + 4096


def test_far_rows_of_few_samples():
    """One long sample has its slots, one for each KV head and 32 sinks, whatever the window."""
    for window in (1, 500):
        one = backward(1, 1 << 20, 8, 128, window, 64) - backward(1, 1 << 20, 8, 128, window, 0)
        assert one >= (16 + 256) * 64 * 128 * 4


@pytest.mark.parametrize("tiles,rows,keys,h_q,h_kv,window,slots", [
    (16, 4096, 4096, 32, 8, 64, 0),               # items of a few key blocks
    (1, 1, 60, 8, 2, 4096, 0),                    # a token of one key block
    (600, 600, 600 * 5000, 8, 2, 4096, 0),        # more tokens than run at once
    (64, 64, 64 * 6000, 32, 8, 4096, 0),          # 512 items of whole tokens
    (32, 32, 32 * 6000, 32, 8, 4096, 512),        # two key ranges for each of 256
    (1, 1, 1 << 20, 8, 2, 1 << 20, 128),          # 64 for each of 2
])
@pytest.mark.parametrize("d", [64, 128])
def test_forward_has_slots_only_where_items_are_cut(tiles, rows, keys, h_q, h_kv, window, slots, d):
    """Beyond what the same call takes with items of a single key block: slots of 128 rows of d + 2
    floats, half as many records of 64 bytes, alignment."""
    def size(w):
        return pl.libra_attn_window_workspace_size(tiles, tiles, rows, keys, h_q, h_kv, d, False,
                                                   window=w, sinks=4)
    more = size(window) - size(1)
    slot = 128 * (d + 2) * 4
    assert slots * slot <= more <= slots * (slot + 32) + 512


@pytest.mark.parametrize("d", [64, 128])
def test_forward_of_a_list_of_long_items(d):
    """As much as libra_attn_fwd asks for, whose items can be cut too."""
    sizes = (16, 2, 4096, 4096, 32, 8, d)
    assert pl.libra_attn_window_workspace_size(*sizes, False, window=4096, sinks=4) \
        == pl.libra_attn_workspace_size(*sizes, False)
