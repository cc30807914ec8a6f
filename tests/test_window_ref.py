"""Pins of window_ref.py on the CPU: its mask against the definition, its values against
softmax written out, its gradients against central differences."""
import math

import torch

import window_ref as ref


def test_visible():
    lengths = [5, 1, 7]
    pos = torch.tensor([0, 3, 4, 5, 6, 12, -1, 13])
    ok = ref.visible(lengths, pos, 14, 3, 1)
    want = [{0}, {0, 1, 2, 3}, {0, 2, 3, 4}, {5}, {6}, {6, 10, 11, 12}, set(), set()]
    assert [set(torch.nonzero(r)[:, 0].tolist()) for r in ok] == want
    causal = ref.visible(lengths, pos, 14, 0, 0)
    assert set(torch.nonzero(causal[5])[:, 0].tolist()) == set(range(6, 13))


def _case(seed=0, n=23, h_q=4, h_kv=2, d=8):
    g = torch.Generator().manual_seed(seed)
    q, k, v, do = (torch.randn((n, h, d), generator=g, dtype=torch.float64)
                   for h in (h_q, h_kv, h_kv, h_q))
    ok = ref.visible([14, 9], torch.arange(n), n, 4, 2)
    cov = torch.ones((n, h_q), dtype=torch.bool)
    cov[5, 1] = cov[17, :] = False
    return q, k, v, do, ok, cov


def test_values():
    q, k, v, _, ok, cov = _case()
    got = ref.attention(q, k, v, ok, cov)
    for r, h in ((0, 0), (13, 3), (20, 2), (5, 0)):
        keys = torch.nonzero(ok[r])[:, 0].tolist()
        s = [float(q[r, h] @ k[j, h // 2]) / math.sqrt(8) for j in keys]
        e = [math.exp(x) for x in s]
        o = sum(w * v[j, h // 2] for w, j in zip(e, keys)) / sum(e)
        assert torch.allclose(got["o"][0][r, h], o, rtol=1e-12, atol=1e-12)
        assert abs(float(got["lse"][0][h, r]) - math.log(sum(e))) < 1e-12
    assert (got["o"][0][17] == 0).all() and (got["o"][0][5, 1] == 0).all()


def test_gradients_against_differences():
    q, k, v, do, ok, cov = _case(1)
    got = ref.attention(q, k, v, ok, cov, dout=do)

    def loss(q, k, v):
        return float((ref.attention(q, k, v, ok, cov)["o"][0] * do).sum())

    g = torch.Generator().manual_seed(2)
    for i, name in enumerate(("dq", "dk", "dv")):
        x = [q, k, v]
        u = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
        eps = 1e-5
        hi, lo = list(x), list(x)
        hi[i], lo[i] = x[i] + eps * u, x[i] - eps * u
        slope = (loss(*hi) - loss(*lo)) / (2 * eps)
        # central differences: eps^2 / 6 of the third derivative, and 2^-53 |loss| / eps
        assert abs(slope - float((got[name][0] * u).sum())) < 1e-7 * (1 + abs(slope))


def test_held_values_take_the_given_o_and_lse():
    """With the exact O and LSE the held form is the gradient itself; with others it is the
    formula P = exp(S - LSE), D = rowsum(dO O)."""
    q, k, v, do, ok, cov = _case(3)
    full = ref.attention(q, k, v, ok, cov, dout=do)
    same = ref.attention(q, k, v, ok, cov, dout=do, held=(full["o"][0], full["lse"][0]))
    for name in ("dq", "dk", "dv"):
        assert torch.allclose(full[name][0], same[name][0], rtol=1e-10, atol=1e-10)
    lse = full["lse"][0] + 0.25
    o = full["o"][0] * 0.5
    got = ref.attention(q, k, v, ok, cov, dout=do, held=(o, lse))
    r, h = 9, 2
    s = (q[r, h] @ k[:, 1].T) / math.sqrt(8)
    p = torch.where(ok[r], torch.exp(s - lse[h, r]), 0.0)
    ds = p * (v[:, 1] @ do[r, h] - do[r, h] @ o[r, h])
    assert torch.allclose(got["dq"][0][r, h], ds @ k[:, 1] / math.sqrt(8), rtol=1e-12, atol=1e-12)
