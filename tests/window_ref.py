"""Windowed attention and its gradients in float64, densely, with bounds on what the
kernels' roundings can change (not collected by pytest).

The kernels multiply in bf16 or fp16 and add in fp32.  Their roundings, each at most half a
step (bf16 2^-8 of the value, fp16 2^-11):

* O = P V / l: P in bf16, the result in bf16: 2^-8 (sum_k p |v| + |O|);
* dQ = scale dS K: dS in bf16, the result in bf16, and D = rowsum(dO O) from the bf16 O:
  2^-8 (scale sum_k |dS| |k| + |dQ|) + scale |dD| sum_k p |k|, |dD| <= 2^-8 sum |dO| |O|;
* dK = scale dS^T Q and dV = P^T dO: dS and P in fp16, the result in bf16 or fp32:
  2^-11 scale sum_q |dS| |q| + 2^-8 |dK|; 2^-11 sum_q p |dO| + 2^-8 |dV|.  dS is formed
  from dP - D, both in fp32, so it carries the sums' errors relative to their terms.

P itself comes from fp32 scores and LSE (relative error of P: their absolute error).  SLACK
covers that and the fp32 sums: 2^-24 for each of some 64 roundings of terms no larger than
the sums of absolute values here, and as much again of scores of magnitude 8 or so; that is
below 2^-14, taken relative to the absolute sums.
"""
import math

import torch

SLACK = 2.0 ** -14
HALF = 2.0 ** -8
HALF16 = 2.0 ** -11


def positions(tiles):
    """Position of every Q row that a tile lists (-1 for others)."""
    rows = max(int(t["q_row"] + t["q_end"] - t["q_begin"]) for t in tiles)
    pos = torch.full((rows,), -1, dtype=torch.int64)
    for t in tiles:
        n = int(t["q_end"] - t["q_begin"])
        pos[int(t["q_row"]):int(t["q_row"]) + n] = torch.arange(int(t["q_begin"]),
                                                              int(t["q_end"]))
    return pos


def coverage(tiles, rows, h_q):
    cov = torch.zeros((rows, h_q), dtype=torch.bool)
    for t in tiles:
        n = int(t["q_end"] - t["q_begin"])
        cov[int(t["q_row"]):int(t["q_row"]) + n, int(t["head_begin"]):int(t["head_end"])] = True
    return cov


def visible(lengths, pos, n_kv, window, sinks):
    """[rows, keys]: may the row at pool position pos attend the key?  window 0: causal."""
    cu = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    cu[1:] = torch.cumsum(torch.tensor(lengths, dtype=torch.int64), 0)
    sample = torch.bucketize(pos, cu, right=True) - 1
    inside = (pos >= 0) & (pos < cu[-1])
    start = cu[sample.clamp(0, len(lengths) - 1)]
    key = torch.arange(n_kv)[None, :]
    p = pos[:, None]
    local = key - start[:, None]
    ok = inside[:, None] & (local >= 0) & (key <= p)
    if window:
        ok &= (key > p - window) | (local < sinks)
    return ok


def attention(q, k, v, ok, cov, scale=None, dout=None, held=None):
    """O and LSE (and with ``dout`` the gradients) of the covered pairs in float64, and the
    bounds above: {name: (value, bound)}.  ``held``: (o, lse) to differentiate with, as an
    8-bit checkpoint does, instead of the exact ones."""
    n_q, h_q, d = q.shape
    n_kv, h_kv, _ = k.shape
    G = h_q // h_kv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    q, k, v = q.double(), k.double(), v.double()
    ok, cov = ok.to(q.device), cov.to(q.device)
    z = dict(dtype=torch.float64, device=q.device)
    O, Ob = torch.zeros((n_q, h_q, d), **z), torch.zeros((n_q, h_q, d), **z)
    LSE = torch.zeros((h_q, n_q), **z)
    if dout is not None:
        dout = dout.double()
        dQ, dQb = torch.zeros((n_q, h_q, d), **z), torch.zeros((n_q, h_q, d), **z)
        dK, dKb, dV, dVb = (torch.zeros((n_kv, h_kv, d), **z) for _ in range(4))
    for h in range(h_q):
        g = h // G
        rows = torch.nonzero(cov[:, h] & ok.any(1))[:, 0]
        if not len(rows):
            continue
        K, V, Q = k[:, g], v[:, g], q[rows, h]
        hide = ~ok[rows]
        used = (~hide).any(0)
        K, V = torch.where(used[:, None], K, 0.0), torch.where(used[:, None], V, 0.0)
        S = ((Q @ K.T) * scale).masked_fill(hide, -math.inf)
        lse = torch.logsumexp(S, 1)
        P = torch.exp(S - lse[:, None])
        o = P @ V
        O[rows, h], LSE[h, rows] = o, lse
        Ob[rows, h] = (HALF + SLACK) * (P @ V.abs()) + HALF * o.abs()
        if dout is None:
            continue
        dO = dout[rows, h]
        if held is not None:
            o, lse = held[0][rows, h].double(), held[1][h, rows].double()
            P = torch.exp(S - lse[:, None])
        D = (dO * o).sum(1, keepdim=True)
        dP = dO @ V.T
        dS = P * (dP - D)
        # sums of absolute values that dP - D is formed from
        terms = P * (dO.abs() @ V.abs().T + (dO.abs() * o.abs()).sum(1, keepdim=True))
        dD = HALF * (dO.abs() * o.abs()).sum(1, keepdim=True) if held is None else 0.0
        dQ[rows, h] = scale * (dS @ K)
        dQb[rows, h] = scale * ((HALF * dS.abs() + dD * P + SLACK * terms) @ K.abs()) \
            + HALF * dQ[rows, h].abs()
        dK[:, g] += scale * (dS.T @ Q)
        dV[:, g] += P.T @ dO
        dKb[:, g] += scale * ((HALF16 * dS.abs() + SLACK * terms).T @ Q.abs())
        dVb[:, g] += (HALF16 + SLACK) * (P.T @ dO.abs())
    out = {"o": (O, Ob), "lse": (LSE, torch.full_like(LSE, SLACK))}
    if dout is not None:
        # dK and dV: the bound before their own rounding (2^-8 |dK| in bf16)
        out.update(dq=(dQ, dQb), dk=(dK, dKb), dv=(dV, dVb))
    return out


def close(name, got, ref, where=None):
    """``got`` within the bound of ``ref`` (value, bound); bf16 dK and dV get their rounding."""
    value, bound = (x.cpu() for x in ref)
    got = got.detach().cpu()
    if got.dtype == torch.bfloat16 and name in ("dk", "dv"):
        bound = bound + HALF * value.abs()
    got = got.double()
    if where is not None:
        got, value, bound = got[where], value[where], bound[where]
    assert torch.isfinite(got).all(), f"{name}: not finite"
    # the smallest normal fp32 number: what underflows may be lost
    over = (got - value).abs() - bound - 2.0 ** -126
    if over.numel():
        at = int(over.argmax())
        assert float(over.max()) <= 0, (
            f"{name}: {float(got.flatten()[at])} against {float(value.flatten()[at])}, bound "
            f"{float(bound.flatten()[at])}, element {at}; {int((over > 0).sum())} of "
            f"{over.numel()} out")
