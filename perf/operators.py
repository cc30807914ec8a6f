"""Operators of windowed attention and of 8-bit activation checkpoints, and their plain forms.

* ``fwd``: attention in which the row at position p of a sample attends the keys
  p - window + 1 .. p of its own sample and the sample's first ``sinks`` keys;
* ``bwd``: its gradients dQ, dK, dV;
* ``ckpt``: activations written in 8 bits (32 elements share a power of two) and read back;
* ``bwd_ckpt``: attention gradients from q, k, v and o held in that form (``window`` 0 is
  plain causal attention);
* ``step``: windowed forward, checkpoint, backward from the checkpoint, as a training step of
  one layer runs.

A case lists packed sample lengths by its ``len_seed`` (long-tailed, median 644 tokens, an
optional long sample last in the pack); with ``batch`` it is a batch of cached sequences of
which each one's newest token attends.  Tensors are drawn from the seed that is passed in.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"

_TILE = np.dtype([("q_begin", "<i8"), ("q_end", "<i8"), ("q_row", "<i8"), ("cost", "<i8"),
                  ("head_begin", "<i4"), ("head_end", "<i4"), ("pack", "<i4"), ("home", "<i4"),
                  ("worker", "<i4"), ("id", "<i4")])


def _case(name, op, **kw):
    c = dict(op=op, tokens=4096, forced=0, sigma=1.5, len_seed=1, h_q=32, h_kv=8, d=128, B=2048,
             H=2, cp=0, batch=0, window=1024, sinks=0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's next token: nothing but launches and latency
        _case("token_1", "fwd", batch=1, tokens=2500, h_q=8, h_kv=2, d=64, sinks=4),
        # the next tokens of a batch of conversations, caches of very different lengths
        _case("tokens_64", "fwd", batch=64, tokens=6000, window=4096, sinks=4, len_seed=6),
        # a short prompt of a small model
        _case("fwd_512_d64", "fwd", tokens=512, h_q=8, h_kv=2, d=64, B=256, H=1, window=128,
              sigma=1.0),
        # a whole 32K pack with the attention shapes of Qwen3-8B, each direction
        _case("fwd_32K", "fwd", tokens=32768, forced=16384, len_seed=2, sinks=4),
        _case("bwd_32K", "bwd", tokens=32768, forced=16384, len_seed=2, sinks=4),
        # a ragged pack: sizes that are multiples of nothing, three heads per KV head
        _case("bwd_ragged_d64", "bwd", tokens=20010, h_q=12, h_kv=4, d=64, B=1237, H=4,
              window=333, sinks=5, len_seed=3),
        # a context-parallel rank's share of a 256K pack (Qwen3-235B-A22B shapes)
        _case("fwd_256K_share", "fwd", tokens=262144, forced=200000, h_q=64, h_kv=4, B=4096, H=1,
              cp=16, window=4096, sinks=128, len_seed=4),
        # the activations of a small layer, and q (or o) of the 32K pack
        _case("ckpt_small", "ckpt", tokens=777, h_q=8, d=64),
        _case("ckpt_32K", "ckpt", tokens=32768),
        # gradients from checkpoints: a small model's causal 4K pack, and the 32K pack
        _case("bwd_ckpt_4K_d64", "bwd_ckpt", tokens=4096, h_q=8, h_kv=2, d=64, B=512, window=0,
              sigma=1.0),
        _case("bwd_ckpt_32K", "bwd_ckpt", tokens=32768, forced=16384, len_seed=2, window=0),
        # one layer of a training step on a 64K pack: the largest
        _case("step_64K", "step", tokens=65536, forced=32768, window=2048, sinks=4, len_seed=5),
    ]


_HEADS = ((1, 1), (2, 1), (4, 1), (4, 4), (6, 3), (8, 2), (8, 8), (12, 4), (16, 2), (32, 4),
          (32, 8), (64, 4))


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(("fwd", "fwd", "bwd", "bwd", "ckpt", "bwd_ckpt", "step"))
    h_q, h_kv = rng.choice(_HEADS)
    c = _case(None, op, sigma=rng.choice((1.0, 1.5, 2.0)), len_seed=rng.randrange(1 << 20), h_q=h_q,
              h_kv=h_kv, d=rng.choice((64, 128, 128)), window=_log_uniform(rng, 1, 8192),
              sinks=rng.choice((0, 0, 1, 4, rng.randint(2, 300))))
    c["H"] = rng.choice([h for h in (1, 2, 4, 8)
                         if h_q % h == 0 and (h_kv % h == 0 or h % h_kv == 0)])
    form = rng.choice(("pack", "pack", "share", "tokens")) if op == "fwd" else "pack"
    if form == "tokens":
        c.update(batch=_log_uniform(rng, 1, 256), tokens=_log_uniform(rng, 16, 16384))
        return c
    if form == "share":
        c["cp"] = rng.choice((4, 8, 16))
        c["B"] = _log_uniform(rng, 256, 4096)
        c["tokens"] = 2 * c["cp"] * c["B"] * rng.randint(1, max(1, 131072 // (2 * c["cp"] * c["B"])))
        c["forced"] = rng.randint(1, int(0.95 * c["tokens"]))
        return c
    c["tokens"] = _log_uniform(rng, 1 if op == "ckpt" else 100, 65536)
    c["B"] = min(_log_uniform(rng, 128, 8192), c["tokens"])
    if rng.random() < 0.5:
        c["forced"] = rng.randint(1, max(1, c["tokens"] // 2))
    if op == "bwd_ckpt" and rng.random() < 0.5:
        c.update(window=0, sinks=0)
    return c


def draw(rng):
    most = work(listed()[-1])["flops"]
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["flops"] <= most and w["bytes"] < 6e9:
            return c


# ---------------------------------------------------------------------------
# samples and tiles

def _lengths(case):
    rng = np.random.default_rng(case["len_seed"])
    if case["batch"]:
        out = case["tokens"] * np.exp(0.7 * rng.standard_normal(case["batch"]))
        return [int(x) for x in np.clip(out, 1, 20000)]
    out, room = [], case["tokens"] - case["forced"]
    while room > 0:
        n = int(round(644 * math.exp(case["sigma"] * rng.standard_normal())))
        n = min(max(n, 1), room)
        out.append(n)
        room -= n
    return out + ([case["forced"]] if case["forced"] else [])


def _tiles(case):
    """(sample lengths, tiles, query rows): blocks of B positions x H head shards, of the
    whole pack, of a rank's two chunks of it, or each cached sequence's last position."""
    lengths = _lengths(case)
    total, rows, out = sum(lengths), 0, []
    if case["batch"]:
        spans = [(int(e) - 1, int(e)) for e in np.cumsum(lengths)]
        shards = 1
    else:
        ranges = [(0, total)]
        if case["cp"]:
            c = total // (2 * case["cp"])
            ranges = [(0, c), (total - c, total)]
        spans = [(b, min(b + case["B"], y)) for x, y in ranges for b in range(x, y, case["B"])]
        shards = case["H"]
    w = case["h_q"] // shards
    for b, e in spans:
        out += [(b, e, rows, 0, s * w, (s + 1) * w, 0, 0, 0, len(out) + s) for s in range(shards)]
        rows += e - b
    return lengths, np.array(out, dtype=_TILE), rows


def _fragments(lengths, tiles):
    """(sample start, first row of the sample, rows, Q row, heads) of every tile x sample."""
    cu = np.concatenate([[0], np.cumsum(lengths)])
    for t in tiles:
        b, e = int(t["q_begin"]), int(t["q_end"])
        j = int(np.searchsorted(cu, b, side="right")) - 1
        while j < len(lengths) and cu[j] < e:
            x, y = max(b, int(cu[j])), min(e, int(cu[j + 1]))
            yield (int(cu[j]), x - int(cu[j]), y - x, int(t["q_row"]) + x - b,
                   int(t["head_begin"]), int(t["head_end"]))
            j += 1


# ---------------------------------------------------------------------------
# plain forms: elementary products, sums and comparisons in fp32

def _bands(s, frag):
    """Chunks of a fragment's rows with the keys that they can attend, whole KV groups at
    once: (rows, heads, KV heads, key indices, allowed [rows, keys])."""
    case = s["case"]
    start, q0, n, row, h0, h1 = frag
    G = case["h_q"] // case["h_kv"]
    W = case["window"] or (1 << 40)
    step = max(1, min((1 << 26) // ((h1 - h0) * (min(W, q0 + n) + case["sinks"] + 256)), max(256, W)))
    for a in range(0, n, step):
        m = min(step, n - a)
        p0 = q0 + a
        lo = max(0, p0 - W + 1)
        keys = torch.cat([torch.arange(min(case["sinks"], lo), device=DEV),
                          torch.arange(lo, p0 + m, device=DEV)])
        p = torch.arange(p0, p0 + m, device=DEV)[:, None]
        ok = (keys <= p) & ((keys > p - W) | (keys < case["sinks"]))
        yield (slice(row + a, row + a + m), slice(h0, h1), slice(h0 // G, (h1 - 1) // G + 1),
               keys + start, ok)


def _grouped(x, groups):
    """[m, heads, d] as [groups, m x heads of a group, d], fp32."""
    m, h, d = x.shape
    return x.float().view(m, groups, h // groups, d).transpose(0, 1).reshape(groups, -1, d)


def _ungrouped(x, m):
    g, mh, d = x.shape
    return x.view(g, m, mh // m, d).transpose(0, 1).reshape(m, -1, d)


def _plain_fwd(s, q, k, v):
    case = s["case"]
    o = torch.zeros(q.shape, dtype=torch.float32, device=DEV)
    lse = torch.zeros((q.shape[1], q.shape[0]), dtype=torch.float32, device=DEV)
    for frag in s["frags"]:
        for rows, heads, kvs, keys, ok in _bands(s, frag):
            m, groups = ok.shape[0], kvs.stop - kvs.start
            qs = _grouped(q[rows, heads], groups)
            ks = k[keys, kvs].float().permute(1, 2, 0).contiguous()
            vs = v[keys, kvs].float().transpose(0, 1).contiguous()
            x = torch.matmul(qs, ks) / math.sqrt(case["d"])
            x = x.view(groups, m, -1, len(keys)).masked_fill_(~ok[None, :, None, :], -math.inf)
            top = x.amax(-1, keepdim=True)
            p = (x - top).exp_()
            total = p.sum(-1, keepdim=True)
            out = torch.matmul(p.view(groups, -1, len(keys)), vs) / total.view(groups, -1, 1)
            o[rows, heads] = _ungrouped(out, m)
            lse[heads, rows] = (top + total.log()).squeeze(-1).permute(0, 2, 1).reshape(-1, m)
    return o, lse


def _plain_bwd(s, q, k, v, o, lse, do):
    scale = 1.0 / math.sqrt(s["case"]["d"])
    dq = torch.zeros(q.shape, dtype=torch.float32, device=DEV)
    dk = torch.zeros(k.shape, dtype=torch.float32, device=DEV)
    dv = torch.zeros(k.shape, dtype=torch.float32, device=DEV)
    for frag in s["frags"]:
        for rows, heads, kvs, keys, ok in _bands(s, frag):
            m, groups = ok.shape[0], kvs.stop - kvs.start
            qs, ds_o = _grouped(q[rows, heads], groups), _grouped(do[rows, heads], groups)
            ks = k[keys, kvs].float().transpose(0, 1).contiguous()
            vs = v[keys, kvs].float().transpose(0, 1).contiguous()
            big = _grouped((do[rows, heads].float() * o[rows, heads].float()).sum(-1, keepdim=True),
                           groups)
            ls = lse[heads, rows].view(groups, -1, m).transpose(1, 2).reshape(groups, -1, 1)
            x = torch.matmul(qs, ks.transpose(1, 2).contiguous()) * scale
            p = (x - ls).exp_().view(groups, m, -1, len(keys))
            p = p.masked_fill_(~ok[None, :, None, :], 0.0).view(groups, -1, len(keys))
            dp = torch.matmul(ds_o, vs.transpose(1, 2).contiguous())
            ds = p * (dp - big)
            dq[rows, heads] = _ungrouped(torch.matmul(ds, ks) * scale, m)
            kk = torch.matmul(ds.transpose(1, 2).contiguous(), qs).transpose(0, 1) * scale
            vv = torch.matmul(p.transpose(1, 2).contiguous(), ds_o).transpose(0, 1)
            dk[keys, kvs] += kk
            dv[keys, kvs] += vv
    return dq, dk, dv


def _power(e):
    """2^e in fp32 for integers -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _plain_pack(x):
    """Groups of 32 along the last axis: integers of at most 127 and the exponent of the group's
    unit, the smallest power of two (2^-126 or more) for which the largest element fits."""
    g = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = g.abs().amax(-1)
    bad = ~torch.isfinite(top)
    e = (torch.frexp(torch.where(bad, 0.0, top))[1].int() - 7).clamp_(min=-126)
    e = e + (torch.round(top * _power(-e)) > 127).int()
    n = torch.round(g * _power(-e)[..., None])
    n = torch.where(bad[..., None], 0.0, n).to(torch.int8)
    return n.view(x.shape), torch.where(bad, 255, e + 127).to(torch.uint8)


def _plain_unpack(n, e):
    unit = torch.where(e == 255, math.nan, _power(e.int().clamp(max=254) - 127))
    return (n.float().view(*e.shape, 32) * unit[..., None]).view(n.shape).to(torch.bfloat16)


# ---------------------------------------------------------------------------

def _randn(g, shape, spread=False):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    step = max(1, (1 << 28) // (shape[1] * shape[2]))
    for a in range(0, shape[0], step):
        x = torch.randn((min(step, shape[0] - a),) + shape[1:], generator=g, device=DEV)
        if spread:   # activations: channels of different size, now and then a large value
            ch = torch.linspace(-2, 2, shape[2], device=DEV).exp()
            x = x * ch * torch.where(torch.rand(x.shape, generator=g, device=DEV) < 0.001, 20.0, 1.0)
        out[a:a + x.shape[0]] = x
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    if case["op"] == "ckpt":
        return {"case": case, "x": _randn(gen, (case["tokens"], case["h_q"], case["d"]), True)}
    lengths, tiles, rows = _tiles(case)
    h_q, h_kv, d, keys = case["h_q"], case["h_kv"], case["d"], sum(lengths)
    cu = np.zeros(len(lengths) + 1, dtype=np.int64)
    cu[1:] = np.cumsum(lengths)
    s = {"case": case, "frags": list(_fragments(lengths, tiles)),
         "q": _randn(gen, (rows, h_q, d)), "k": _randn(gen, (keys, h_kv, d)),
         "v": _randn(gen, (keys, h_kv, d)), "cu": torch.from_numpy(cu).to(DEV),
         "tiles": torch.from_numpy(tiles.view(np.uint8).copy()).to(DEV)}
    if case["op"] != "fwd":
        s["do"] = _randn(gen, (rows, h_q, d))
        if case["op"] != "step":
            o, s["lse"] = _plain_fwd(s, s["q"], s["k"], s["v"])
            s["o"] = o.to(torch.bfloat16)
        if case["op"] == "bwd_ckpt":
            for name in "qkvo":
                s[name] = _plain_pack(s[name])
    if own:
        import paper_2607_23250_amd as pl
        s["pl"] = pl
        sizes = (len(tiles), len(lengths), rows, keys, h_q, h_kv, d)
        mask = dict(window=case["window"], sinks=case["sinks"])
        need = 0
        if case["op"] in ("fwd", "step"):
            need = pl.libra_attn_window_workspace_size(*sizes, False, **mask)
        if case["op"] == "bwd":
            need = pl.libra_attn_window_workspace_size(*sizes, True, **mask)
        if case["op"] in ("bwd_ckpt", "step"):
            need = max(need, pl.libra_attn_bwd_ckpt8_workspace_size(*sizes, **mask))
        s["ws"] = pl.alloc_workspace(need, DEV)
        # buffers that a program keeps over its layers
        s["out"] = torch.zeros((rows, h_q, d), dtype=torch.bfloat16, device=DEV)
        s["lse_out"] = torch.zeros((h_q, rows), dtype=torch.float32, device=DEV)
        if case["op"] != "fwd":
            s["dq"] = torch.zeros_like(s["out"])
            s["dk"] = torch.zeros((keys, h_kv, d), dtype=torch.bfloat16, device=DEV)
            s["dv"] = torch.zeros_like(s["dk"])
    return s


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "ckpt":
        if own:
            import paper_2607_23250_amd as pl
            n, e = pl.libra_ckpt8_pack(s["x"])
            return {"x": pl.libra_ckpt8_unpack(n, e)}
        return {"x": _plain_unpack(*_plain_pack(s["x"]))}
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    pl, case, op = s["pl"], s["case"], s["case"]["op"]
    mask = dict(window=case["window"], sinks=case["sinks"])
    q, k, v = s["q"], s["k"], s["v"]
    if op in ("fwd", "step"):
        o, lse = pl.libra_attn_window_fwd(q, k, v, s["cu"], s["tiles"], o=s["out"],
                                          lse=s["lse_out"], workspace=s["ws"], **mask)
    if op == "fwd":
        return {"o": o, "lse": lse}
    grads = dict(dq=s["dq"], dk=s["dk"], dv=s["dv"], workspace=s["ws"], **mask)
    if op == "bwd":
        dq, dk, dv = pl.libra_attn_window_bwd(q, k, v, s["o"], s["lse"], s["do"], s["cu"],
                                              s["tiles"], **grads)
    elif op == "bwd_ckpt":
        dq, dk, dv = pl.libra_attn_bwd_ckpt8(q, k, v, s["o"], s["lse"], s["do"], s["cu"],
                                             s["tiles"], **grads)
    else:
        held = [pl.libra_ckpt8_pack(x) for x in (q, k, v, o)]
        dq, dk, dv = pl.libra_attn_bwd_ckpt8(*held, lse, s["do"], s["cu"], s["tiles"], **grads)
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    return {"dq": dq, "dk": dk, "dv": dv}


def _run_plain(s):
    op, b16 = s["case"]["op"], torch.bfloat16
    if op in ("fwd", "step"):
        o, lse = _plain_fwd(s, s["q"], s["k"], s["v"])
        o = o.to(b16)
    if op == "fwd":
        return {"o": o, "lse": lse}
    if op == "bwd":
        dq, dk, dv = _plain_bwd(s, s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"])
    elif op == "bwd_ckpt":
        q, k, v, o = (_plain_unpack(*s[name]) for name in "qkvo")
        dq, dk, dv = _plain_bwd(s, q, k, v, o, s["lse"], s["do"])
    else:
        held = [_plain_unpack(*_plain_pack(x)) for x in (s["q"], s["k"], s["v"], o)]
        dq, dk, dv = _plain_bwd(s, *held, lse, s["do"])
        return {"o": o, "lse": lse, "dq": dq.to(b16), "dk": dk.to(b16), "dv": dv.to(b16)}
    return {"dq": dq.to(b16), "dk": dk.to(b16), "dv": dv.to(b16)}


# ---------------------------------------------------------------------------

def _pairs_and_keys(case, lengths, tiles):
    """(attended (row, head, key) triples, (row, head) pairs, (key, KV head) pairs reached)."""
    G = case["h_q"] // case["h_kv"]
    W = case["window"] or (1 << 40)
    pairs = rows = 0
    reach = {}
    for start, q0, n, _, h0, h1 in _fragments(lengths, tiles):
        p = np.arange(q0, q0 + n)
        lo = np.maximum(0, p - W + 1)
        pairs += int((p + 1 - lo + np.minimum(case["sinks"], lo)).sum()) * (h1 - h0)
        rows += n * (h1 - h0)
        for g in range(h0 // G, (h1 - 1) // G + 1):
            first = int(lo[0])
            reach.setdefault((start, g), []).extend(
                [(0, min(case["sinks"], q0 + n)), (first, q0 + n)])
    keys = 0
    for spans in reach.values():
        end = 0
        for a, b in sorted(spans):
            keys += max(0, b - max(a, end))
            end = max(end, b)
    return pairs, rows, keys


def work(case):
    d = case["d"]
    if case["op"] == "ckpt":
        # bf16 in, 8 bits and an exponent for 32 out; the same in, bf16 out
        n = case["tokens"] * case["h_q"] * d
        return {"bytes": int(2 * n * (2 + 33 / 32)), "flops": 0}
    lengths, tiles, _ = _tiles(case)
    pairs, rows, keys = _pairs_and_keys(case, lengths, tiles)
    all_kv = sum(lengths) * case["h_kv"] * d
    fwd = rows * (2 * d * 2 + 4) + keys * 2 * d * 2
    if case["op"] == "fwd":
        return {"bytes": fwd, "flops": 4 * d * pairs}
    if case["op"] == "bwd":   # q, o, dO and lse in, dQ out; K and V in, dK and dV out
        return {"bytes": rows * (4 * d * 2 + 4) + keys * 2 * d * 2 + 2 * all_kv * 2,
                "flops": 10 * d * pairs}
    held = 33 / 32
    bwd = rows * (2 * d * held + 2 * d * 2 + 4) + keys * 2 * d * held
    if case["op"] == "bwd_ckpt":
        return {"bytes": int(bwd + 2 * all_kv * 2), "flops": 10 * d * pairs}
    pack = (2 * rows * d + 2 * all_kv) * (2 + held)
    return {"bytes": int(fwd + pack + bwd + 2 * all_kv * 2), "flops": 14 * d * pairs}


def _exact_pack(x):
    """The values that 8 bits hold of x, in fp64, from the definition: the unit of 32 elements is
    the smallest power of two, 2^-126 or more, in which their largest rounds to at most 127."""
    g = x.double().reshape(-1, 32)
    top = g.abs().max(1, keepdim=True).values
    unit = torch.full_like(top, 2.0 ** -126)
    for e in range(-125, 122):   # one step at a time: fits or doubles
        unit = torch.where((top / unit).round() > 127, torch.full_like(top, 2.0 ** e), unit)
    return ((g / unit).round() * unit).reshape(x.shape)


def exact(case, seed):
    """Softmax attention, its gradients and the 8-bit values in float64, head by head."""
    op = case["op"]
    s = prepare(case, seed)
    if op == "ckpt":
        return {"x": _exact_pack(s["x"])}
    h_q, h_kv, d, W, S = (case[n] for n in ("h_q", "h_kv", "d", "window", "sinks"))
    W = W or (1 << 40)
    lengths, tiles, rows = _tiles(case)
    if _pairs_and_keys(case, lengths, tiles)[0] > 2e10:
        return None   # over 20 seconds in 64 bits
    G, scale = h_q // h_kv, d ** -0.5
    f64 = dict(dtype=torch.float64, device=DEV)

    def blocks():
        """(rows, head, KV head, first and one past the last of the far and of the near keys,
        which of them count) of 1024 rows or fewer and one query head."""
        for start, q0, n, row, h0, h1 in _fragments(lengths, tiles):
            for a in range(0, n, 1024):
                m = min(1024, n - a)
                near = max(0, q0 + a + 1 - W)
                far = min(S, near)
                at = torch.arange(q0 + a, q0 + a + m, device=DEV).unsqueeze(1)
                pos = torch.arange(near, q0 + a + m, device=DEV).unsqueeze(0)
                hide = torch.zeros((m, far + pos.shape[1]), dtype=torch.bool, device=DEV)
                hide[:, far:] = (pos > at) | ((at - pos >= W) & (pos >= S))
                for h in range(h0, h1):
                    yield (slice(row + a, row + a + m), h, h // G, slice(start, start + far),
                           slice(start + near, start + q0 + a + m), hide)

    def scores(q, k, b):
        r, h, g, far, near, hide = b
        ks = torch.cat([k[far, g], k[near, g]]).double()
        x = (q[r, h].double() * scale) @ ks.T
        x[hide] = -math.inf
        return x, ks

    out = {}
    if op in ("fwd", "step"):
        o, lse = torch.zeros((rows, h_q, d), **f64), torch.zeros((h_q, rows), **f64)
        for b in blocks():
            r, h, g, far, near, _ = b
            x, _ = scores(s["q"], s["k"], b)
            lse[h, r] = torch.logsumexp(x, 1)
            o[r, h] = torch.softmax(x, 1) @ torch.cat([s["v"][far, g], s["v"][near, g]]).double()
        out.update(o=o, lse=lse)
    if op == "fwd":
        return out
    if op == "bwd":
        q, k, v, o, lse = s["q"], s["k"], s["v"], s["o"], s["lse"]
    elif op == "step":
        q, k, v, o = (_exact_pack(x) for x in (s["q"], s["k"], s["v"], o.to(torch.bfloat16)))
    else:
        q, k, v, o = ((n.double().reshape(-1, 32) *
                       torch.exp2(e.double().reshape(-1, 1) - 127)).reshape(n.shape)
                      for n, e in (s["q"], s["k"], s["v"], s["o"]))
        lse = s["lse"]
    dq = torch.zeros((rows, h_q, d), **f64)
    dk, dv = (torch.zeros((sum(lengths), h_kv, d), **f64) for _ in range(2))
    for b in blocks():
        r, h, g, far, near, _ = b
        x, ks = scores(q, k, b)
        p = (x - lse[h, r].double().unsqueeze(1)).exp()
        vs = torch.cat([v[far, g], v[near, g]]).double()
        dos = s["do"][r, h].double()
        ds = p * (dos @ vs.T - (dos * o[r, h].double()).sum(1, keepdim=True)) * scale
        dq[r, h] = ds @ ks
        gk, gv = ds.T @ q[r, h].double(), p.T @ dos
        c = far.stop - far.start
        dk[far, g] += gk[:c]
        dk[near, g] += gk[c:]
        dv[far, g] += gv[:c]
        dv[near, g] += gv[c:]
    out.update(dq=dq, dk=dk, dv=dv)
    return out
