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
