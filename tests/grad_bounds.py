"""What large scores and a caller's softmax_scale add to the bounds of window_ref.py (not
collected by pytest).

* P: window_ref.py counts scores of magnitude 8 or so.  A score is a sum of d products in fp32,
  with -LSE / scale as one more term, so it is off by at most d + 16 roundings of 2^-24 of its
  terms' absolute sum, scale sum |q| |k| + |LSE|, and |LSE| is at most as much again and ln n;
  P is off by that in relation to itself, and so are dS (in relation to the terms of dP - D) and,
  through the sums over a row that correct O, LSE and D, everything once more: four times in all.
* fp16 numbers below 2^-14 lie 2^-24 apart, so P, dS and the copies of q, k, v and dout are also
  off by up to 2^-25 in the units of their scales: those bring max |dout| and max |v| to [1, 2)
  and max |q| and max |k| below 8, or lower for a very small softmax_scale, by `down`.  (The
  windowed dQ forms its dS times 16.)
* fp32 and bf16 numbers below 2^-126 may become zero: a P, which loses P (dP - D), or a dS, each
  times scale |k| in dQ.  (dK and dV lose less than by the second point.)
"""
import math

import torch

import window_ref as ref

STEP = 2.0 ** -25
SLACK = ref.SLACK


def score_error(q, k, scale, pairs):
    """Of P, relative: the largest over the pairs [rows, heads, keys that a row attends]."""
    ok, cov = pairs
    G = q.shape[1] // k.shape[1]
    most = 0.0
    for h in range(q.shape[1]):
        rows = torch.nonzero(cov[:, h] & ok.any(1))[:, 0]
        s = (q[rows, h].double().abs() @ k[:, h // G].double().abs().T) * ok[rows]
        most = max(most, float(s.max()) * scale) if len(rows) else most
    return 4 * (q.shape[2] + 16) * 2.0 ** -24 * (2 * most + math.log(k.shape[0]))


def underflow(q, k, v, do, pairs, scale, lse, down=1.0):
    """The bounds of the second and third points; lse [heads, rows]."""
    ok, cov = pairs
    n_kv, h_kv, d = k.shape
    G = q.shape[1] // h_kv
    q, k, v, do, lse = (x.double() for x in (q, k, v, do, lse))
    top_q, top_k = (max(1.0, float(x.abs().max()) / 4) * down for x in (q, k))
    top_o, top_v = float(do.abs().max()), float(v.abs().max())
    dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64) for x in (q, k, v))
    for h in range(q.shape[1]):
        g = h // G
        rows = torch.nonzero(cov[:, h] & ok.any(1))[:, 0]
        seen = ok[rows].double()
        Q, dO = q[rows, h], do[rows, h]
        S = ((Q @ k[:, g].T) * scale).masked_fill(~ok[rows], -math.inf)
        P = torch.exp(S - lse[h, rows, None])
        size = dO.abs() @ v[:, g].abs().T + d * top_o * top_v   # |dP| + |D| at most
        dv[:, g] += STEP * (seen.T @ dO.abs() + P.sum(0)[:, None] * top_o)
        dk[:, g] += STEP * scale * (
            (top_o * top_v * (seen + 2 * d * P)).T @ Q.abs()
            + (P * size).sum(0)[:, None] * top_q)
        dq[rows, h] = scale * (
            ((2.0 ** -126 * (1 + size) + STEP / 16 * top_o * top_v) * seen + STEP * 2 * d * top_o
             * top_v * P) @ k[:, g].abs() + STEP * top_k * (P * size).sum(1, keepdim=True))
    return {"dq": dq, "dk": dk, "dv": dv}


def gradients(monkeypatch, q, k, v, do, pairs, scale, lse, held=None, down=1.0):
    """window_ref.attention of these (CPU) tensors with all three points in the bounds.  ``held``:
    its (o, lse); ``lse``: what P is formed with."""
    monkeypatch.setattr(ref, "SLACK", SLACK + score_error(q, k, scale, pairs))
    want = ref.attention(q, k, v, *pairs, scale=scale, dout=do, held=held)
    for name, more in underflow(q, k, v, do, pairs, scale, lse, down).items():
        want[name] = (want[name][0], want[name][1] + more)
    return want
