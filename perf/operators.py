"""Measured cases of the operators a rotated, quantised model runs on: the RMSNorm that adds the residual and quantises
per token, the append of rotated keys and quantised keys and values to a paged cache, and the attention that reads it.

`own = False` computes them from elementary torch operations, `own = True` calls the library.  Cases are plain dicts;
`kind` names the operator.
"""
import math

import torch

own = False

DEV = "cuda:0"
ROPE_BASE = 500000.0


def listed():
    return [
        # --- norm: widths are the hidden and feed-forward widths of the benchmark's workloads (4096, 8192, 14336)
        # one token of one request: latency
        dict(name="norm_token", kind="norm", rows=1, d=4096, pad=0, dtype="bf16", residual=True, gain=False, bits=8,
             clip=1.0, out="codes"),
        # a decode step of an odd batch whose rows are a slice of a wider buffer
        dict(name="norm_batch", kind="norm", rows=257, d=8192, pad=64, dtype="bf16", residual=True, gain=True, bits=8,
             clip=0.98, out="codes"),
        # the prompts of a large prefill step
        dict(name="norm_prompt", kind="norm", rows=16384, d=4096, pad=0, dtype="bf16", residual=True, gain=False,
             bits=8, clip=1.0, out="codes"),
        # simulated 4-bit activations in float32, as a quality evaluation runs them
        dict(name="norm_simulated", kind="norm", rows=4099, d=14336, pad=0, dtype="f32", residual=False, gain=False,
             bits=4, clip=0.98, out="values"),
        # --- append: one decode step of 64 requests, keys behind an online Hadamard rotation
        dict(name="append_tokens", kind="append", seqs=64, rows=1, length=4096, q_heads=32, heads=8, head_dim=128,
             page=64, bits=4, asym=True, clip=1.0, hadamard=True, rope=True, dtype="bf16", ragged=True, pad=0),
        # a prefill step over a few prompts of uneven length, 4-bit
        dict(name="append_prompts", kind="append", seqs=5, rows=6000, length=6000, q_heads=32, heads=8, head_dim=128,
             page=64, bits=4, asym=True, clip=1.0, hadamard=True, rope=True, dtype="bf16", ragged=True, pad=0),
        # chunks on top of what is cached, 64-wide heads, 8-bit symmetric, small pages, float32 projections
        dict(name="append_chunks", kind="append", seqs=16, rows=511, length=9000, q_heads=24, heads=24, head_dim=64,
             page=16, bits=8, asym=False, clip=0.95, hadamard=False, rope=True, dtype="f32", ragged=True, pad=5),
        # --- attend, single tokens: one request
        dict(name="token_one", kind="attend", seqs=1, rows=1, length=1500, q_heads=32, heads=8, head_dim=128, page=64,
             bits=4, window=0, ragged=False, pad=0, lse=False),
        # a decode step of a batch of uneven lengths
        dict(name="token_batch", kind="attend", seqs=64, rows=1, length=8192, q_heads=64, heads=8, head_dim=128,
             page=64, bits=4, window=0, ragged=True, pad=0, lse=True),
        # a few very long requests, 8-bit
        dict(name="token_long", kind="attend", seqs=3, rows=1, length=131072, q_heads=32, heads=8, head_dim=128,
             page=128, bits=8, window=0, ragged=True, pad=0, lse=False),
        # a whole prompt
        dict(name="prompt_whole", kind="attend", seqs=1, rows=8192, length=8192, q_heads=32, heads=8, head_dim=128,
             page=64, bits=4, window=0, ragged=False, pad=0, lse=False),
        # chunks of several prompts behind what is cached, sliding window, 64-wide heads
        dict(name="prompt_chunks", kind="attend", seqs=6, rows=700, length=5000, q_heads=24, heads=6, head_dim=64,
             page=16, bits=8, window=2048, ragged=True, pad=3, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["norm", "append", "attend"])
    if kind == "norm":
        d = rng.choice([128 * rng.randint(1, 112), 8 * rng.randint(5, 1200), rng.randint(33, 9001)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(kind=kind, rows=_log(rng, 1, 6.0e7 / d), d=d, pad=rng.choice([0, 0, 8, 3]), dtype=dtype,
                    residual=rng.random() < 0.7, gain=rng.random() < 0.5, bits=rng.choice([4, 8]),
                    clip=rng.choice([1.0, 0.98, 0.9]), out=rng.choice(["codes", "values"]))
    head_dim = rng.choice([64, 128, 128])
    heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 3, 4, 5, 8, 16])
    page = rng.choice([16, 32, 64, 128])
    bits = rng.choice([4, 8])
    if kind == "append":
        seqs = _log(rng, 1, 100)
        rows = _log(rng, 1, min(6000, max(1, int(2.0e8 / (seqs * heads * (group + 2) * head_dim)))))
        return dict(kind=kind, seqs=seqs, rows=rows, length=rows + _log(rng, 1, 4000) - 1, q_heads=heads * group,
                    heads=heads, head_dim=head_dim, page=page, bits=bits, asym=rng.random() < 0.7,
                    clip=rng.choice([1.0, 0.95]), hadamard=rng.random() < 0.5, rope=rng.random() < 0.8,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.7, pad=rng.choice([0, 0, 7]))
    if rng.random() < 0.5:  # single tokens, or a few tokens that are verified together
        rows = rng.choice([1, 1, 1, 2, 5])
        seqs = _log(rng, 1, 128)
        length = _log(rng, rows, max(rows, min(131072, int(4.0e5 * 8 / (seqs * heads)))))
    else:
        rows = _log(rng, 17, 4096)
        seqs = _log(rng, 1, max(1, min(12, 8192 // rows)))
        length = _log(rng, rows, max(rows, min(16384, int(1.5e9 / (seqs * heads * group * rows)))))
    return dict(kind=kind, seqs=seqs, rows=rows, length=length, q_heads=heads * group, heads=heads, head_dim=head_dim,
                page=page, bits=bits, window=rng.choice([0, 0, 0, _log(rng, 32, 8192)]), ragged=rng.random() < 0.7,
                pad=rng.choice([0, 0, 3]), lse=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------- sequences of a case
def _sizes(case):
    """Rows and lengths of every sequence (host lists), the same for every seed: (rows, lengths)."""
    n = case["seqs"]
    if not case["ragged"]:
        return [case["rows"]] * n, [case["length"]] * n
    rows, lens = [], []
    for s in range(n):  # uneven, the first one full; the third has rows only, the fourth is one token
        f = 1.0 if s == 0 else ((s * 37 + 11) % 97 + 1) / 98.0
        r = max(1, int(case["rows"] * (1.0 if s == 0 else ((s * 53 + 29) % 89 + 1) / 90.0)))
        if s == 3:
            r = 1
        past = int((case["length"] - case["rows"]) * f)
        rows.append(r)
        lens.append(r if s == 2 else r + past)
    return rows, lens


def _visible(case):
    """(row, key) pairs that the mask leaves, per query head."""
    total = 0
    for r, n in zip(*_sizes(case)):
        w = case["window"] or n
        for p in (range(n - r, n) if r <= 64 else ()):
            total += min(p + 1, w)
        if r > 64:
            lo, hi = n - r, n - 1
            full = max(0, hi - max(lo, w - 1) + 1)
            part = (hi - lo + 1) - full
            total += full * w + part * (lo + 1) + part * (part - 1) // 2
    return total


def work(case):
    """What one pass has to read, write and compute."""
    if case["kind"] == "norm":
        n, e = case["rows"] * case["d"], 2 if case["dtype"] == "bf16" else 4
        b = n * e * (3 if case["residual"] else 1) + case["d"] * (4 if case["gain"] else 0) + case["rows"] * 4
        b += n * (1 if case["out"] == "codes" else 2)
        return {"bytes": b, "flops": 8 * n}
    rows, lens = _sizes(case)
    N, T = sum(rows), sum(lens)
    hd, h, hq = case["head_dim"], case["heads"], case["q_heads"]
    held = hd * case["bits"] / 8 + 8  # one token of one head: codes and the pair (scale, shift)
    if case["kind"] == "append":
        e = 2 if case["dtype"] == "bf16" else 4
        b = N * (hq + 2 * h) * hd * e + N * (hq + 2 * h) * hd * 2 + N * 2 * h * held
        b += N * hd * 4 if case["rope"] else 0
        return {"bytes": b, "flops": N * (hq + 2 * h) * hd * 12}
    keys = sum(min(n, r + case["window"]) if case["window"] else n for r, n in zip(rows, lens))
    b = 2 * N * hq * hd * 2 + keys * h * 2 * held + (N * hq * 4 if case["lse"] else 0)
    return {"bytes": b, "flops": 4 * _visible(case) * hq * hd}


# ------------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _strided(t, pad):
    """The same values as a slice of a buffer whose rows are `pad` elements longer."""
    if not pad:
        return t.contiguous()
    wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def _channels(g, rows, d, factor):
    """Activations with a few channels that are `factor` times larger, as calibration sees them."""
    x = _randn(g, rows, d)
    at = torch.randperm(d, generator=g, device=DEV)[: max(1, d // 256)]
    x[:, at] *= factor
    return x


def _rope_table(positions, head_dim):
    """[positions][head_dim / 2][2]: cosine and sine, from angles in 64 bits."""
    i = torch.arange(head_dim // 2, device=DEV, dtype=torch.float64)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * ROPE_BASE ** (-2.0 * i / head_dim)
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def _paged(case, g, lens):
    """Page table (pages in no order), and the number of pages."""
    page = case["page"]
    most = max(1, -(-max(lens) // page))
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(case["seqs"], most, dtype=torch.int32)
    at = 0
    host = order.cpu()
    for s, n in enumerate(need):
        table[s, :n] = host[at : at + n]
        at += n
    return table.to(DEV), pages


_context = None


def _ctx():
    """A program keeps one context."""
    global _context
    if _context is None:
        from paper_2503_01483_b200 import kurtail

        _context = kurtail.Context(DEV)
    return _context


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=case)
    if case["kind"] == "norm":
        t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        n, d = case["rows"], case["d"]
        st["x"] = _strided(_channels(g, n, d, 20.0).to(t), case["pad"])
        st["residual"] = _strided((_channels(g, n, d, 20.0) * 3).to(t), case["pad"]) if case["residual"] else None
        st["sum"] = torch.empty_like(st["residual"]) if case["residual"] else None
        st["gain"] = 1.0 + 0.2 * _randn(g, d) if case["gain"] else None
        st["codes"] = torch.empty(n, d, dtype=torch.int8, device=DEV) if case["out"] == "codes" else None
        st["scales"] = torch.empty(n, dtype=torch.float32, device=DEV)
        st["values"] = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
        if own:
            _ctx()
        return st
    rows, lens = _sizes(case)
    hd, h, hq = case["head_dim"], case["heads"], case["q_heads"]
    N = sum(rows) + case["pad"]
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    st["row_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    st["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st["page_table"], pages = _paged(case, g, lens)
    st["max_rows"], st["max_length"] = max(rows), max(lens)
    held = hd * case["bits"] // 8
    shape = (pages, h, case["page"])
    if case["kind"] == "append":
        t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        qkv = _randn(g, N, (hq + 2 * h) * hd)  # one fused projection; a few key channels carry large values
        qkv[:, hq * hd : (hq + h) * hd].view(N, h, hd)[:, :, 3 :: hd // 2] *= 8.0
        qkv = qkv.to(t)
        st["q"], st["k"], st["v"] = qkv[:, : hq * hd], qkv[:, hq * hd : (hq + h) * hd], qkv[:, (hq + h) * hd :]
        st["rope"] = _rope_table(max(lens), hd) if case["rope"] else None
        for x in "kv":
            st[x + "_codes"] = torch.zeros(*shape, held, dtype=torch.uint8, device=DEV)
            st[x + "_steps"] = torch.zeros(*shape, 2, device=DEV)
            st[x + "_values"] = torch.zeros(N, h * hd, dtype=torch.bfloat16, device=DEV)
        st["q_out"] = torch.zeros(N, hq * hd, dtype=torch.bfloat16, device=DEV)
    else:
        top = 2 ** case["bits"] - 1
        for x in "kv":  # what an append would have left: per token and head, its range in steps from its minimum
            y = _randn(g, *shape, hd)
            y += 0.5 * _randn(g, h, 1, hd)
            low = y.amin(-1, keepdim=True)
            step = (y.amax(-1, keepdim=True) - low) / top
            c = torch.round((y - low) / step).clamp_(0, top).to(torch.uint8)
            st[x + "_steps"] = torch.cat((step, low), -1).contiguous()
            st[x + "_codes"] = (c[..., 0::2] | (c[..., 1::2] << 4)).contiguous() if case["bits"] == 4 else c
            del y
        st["q"] = (1.2 * _randn(g, N, hq * hd)).bfloat16()
        st["out"] = torch.zeros(N, hq * hd, dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros(N, hq, device=DEV) if case["lse"] else None
    if own:
        from paper_2503_01483_b200 import kurtail

        st["cache"] = kurtail.KvCache(st["k_codes"], st["v_codes"], st["k_steps"], st["v_steps"], case["bits"])
        st["batch"] = _ctx().kv_batch(st["cache"], hq, st["row_starts"], st["lengths"], st["page_table"],
                                      st["max_rows"], st["max_length"])
    return st


# ---------------------------------------------------------------------------------------------------- the plain forms
def _over(x, by):
    """x / by with the division's own rounding (by a number, torch multiplies with the reciprocal)."""
    return x / torch.full_like(x, by)


def _norm_plain(st):
    c = st["case"]
    h = st["x"].float()
    if st["residual"] is not None:
        st["sum"].copy_(h + st["residual"].float())
        h = st["sum"].float()
    # the sum of squares and the root in 64 bits, then one float32 factor; from there on float32, operation by operation
    factor = (1.0 / torch.sqrt(h.double().square().mean(1, keepdim=True) + 1e-6)).float()
    y = h * factor
    if st["gain"] is not None:
        y = y * st["gain"]
    top = 2 ** (c["bits"] - 1) - 1
    s = _over(y.abs().amax(1, keepdim=True) * c["clip"], top)
    q = torch.where(s > 0, torch.round(y / s).clamp(-top, top), torch.zeros_like(y))
    st["values"].copy_(q * s)
    return {"values": st["values"], "scales": s[:, 0], "sum": st["sum"]}


def _sequence_of_rows(st, n):
    """Sequence and position of every row of the batch; rows behind the last sequence have none."""
    r = torch.arange(n, device=DEV, dtype=torch.int32)
    s = torch.searchsorted(st["row_starts"], r, right=True) - 1
    ok = s < st["lengths"].numel()
    s = s.clamp(max=st["lengths"].numel() - 1)
    pos = st["lengths"][s] - (st["row_starts"][s + 1] - r)
    return s, pos, ok


def _rotated_plain(x, pos, rope, hadamard):
    """Rotary positions (pairs half a head apart), then the normalised Hadamard rotation in log2 stages,
    the widest first."""
    hd = x.shape[-1]
    if rope is not None:
        t = rope[pos][:, None]
        c, s = t[..., 0], t[..., 1]
        a, b = x[..., : hd // 2], x[..., hd // 2 :]
        x = torch.cat((a * c - b * s, b * c + a * s), -1)
    if hadamard:
        x = _hadamard_stages(x, hd // 2)
    return x


def _hadamard_stages(x, w):
    hd = x.shape[-1]
    if w == 0:
        return x * (1.0 / math.sqrt(hd))
    p = x.reshape(*x.shape[:-1], hd // (2 * w), 2, w)
    a, b = p[..., 0, :], p[..., 1, :]
    return _hadamard_stages(torch.stack((a + b, a - b), -2).reshape(x.shape), w // 2)


def _quantised_plain(y, c):
    """Codes (from zero upwards), step and shift of every row of y."""
    clip = c["clip"]
    if c["asym"]:
        top = 2 ** c["bits"] - 1
        b = y.amin(-1, keepdim=True) * clip
        s = _over(y.amax(-1, keepdim=True) * clip - b, top)
        q = torch.where(s > 0, torch.round((y - b) / s).clamp(0, top), torch.zeros_like(y))
        return q, s, b
    half = 2 ** (c["bits"] - 1)
    s = _over(y.abs().amax(-1, keepdim=True) * clip, half - 1)
    q = torch.where(s > 0, torch.round(y / s).clamp(1 - half, half - 1), torch.zeros_like(y))
    return q + half, s, -s * half


def _put_plain(st, name, y, s, pos, ok):
    c = st["case"]
    q, step, shift = _quantised_plain(y, c)
    n, h, hd = y.shape
    page = st["page_table"][s, (pos // c["page"]).long()][ok].long()[:, None]
    head, at = torch.arange(h, device=DEV)[None], (pos % c["page"])[ok][:, None]
    u = q.to(torch.uint8)[ok]
    st[name + "_codes"][page, head, at] = u[..., 0::2] | (u[..., 1::2] << 4) if c["bits"] == 4 else u
    st[name + "_steps"][page, head, at] = torch.cat((step, shift), -1)[ok]
    st[name + "_values"][ok] = (q * step + shift).bfloat16().reshape(n, h * hd)[ok]


def _append_plain(st):
    c = st["case"]
    n, hd = st["q"].shape[0], c["head_dim"]
    s, pos, ok = _sequence_of_rows(st, n)
    pos = pos.clamp(min=0)
    q = _rotated_plain(st["q"].float().reshape(n, -1, hd), pos, st["rope"], c["hadamard"])
    st["q_out"][ok] = q.bfloat16().reshape(n, -1)[ok]
    _put_plain(st, "k", _rotated_plain(st["k"].float().reshape(n, -1, hd), pos, st["rope"], c["hadamard"]), s, pos, ok)
    _put_plain(st, "v", st["v"].float().reshape(n, -1, hd), s, pos, ok)
    return {x: st[x] for x in ("q_out", "k_values", "v_values", "k_steps", "v_steps")}


def _cached_plain(st, name):
    """[sequences][heads][tokens][head_dim] float32: what the cache stands for."""
    c = st["case"]
    u = st[name + "_codes"][st["page_table"].long()]
    if c["bits"] == 4:
        u = torch.stack((u & 15, u >> 4), -1).flatten(-2)
    step = st[name + "_steps"][st["page_table"].long()]
    y = u.float() * step[..., :1] + step[..., 1:]
    return y.transpose(1, 2).flatten(2, 3)


def _attend_plain(st):
    c = st["case"]
    hd, h, hq = c["head_dim"], c["heads"], c["q_heads"]
    n, S, R = st["q"].shape[0], c["seqs"], st["max_rows"]
    K, V = _cached_plain(st, "k"), _cached_plain(st, "v")
    L = K.shape[2]
    r = torch.arange(R, device=DEV)
    rows = st["row_starts"][:-1, None] + r  # [S][R]
    there = rows < st["row_starts"][1:, None]
    rows = torch.where(there, rows, 0).long()
    q = st["q"].float()[rows].reshape(S, R, h, hq // h, hd).permute(0, 2, 3, 1, 4).reshape(S, h, -1, hd)
    scores = (q @ K.transpose(-1, -2)).mul_(1.0 / math.sqrt(hd)).reshape(S, h, hq // h, R, L)
    pos = (st["lengths"] - (st["row_starts"][1:] - st["row_starts"][:-1]))[:, None] + r
    j = torch.arange(L, device=DEV)
    hidden = j > pos[..., None]
    if c["window"]:
        hidden = hidden | (j <= pos[..., None] - c["window"])
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(S, h, -1, L) @ V).reshape(S, h, hq // h, R, hd) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log())[..., 0]
    st["out"][rows[there]] = o.permute(0, 3, 1, 2, 4).reshape(S, R, hq * hd)[there].bfloat16()
    if st["lse"] is not None:
        st["lse"][rows[there]] = lse.permute(0, 3, 1, 2).reshape(S, R, hq)[there]
    return {"out": st["out"], "lse": st["lse"]}


def run(st):
    c = st["case"]
    if not own:
        return {"norm": _norm_plain, "append": _append_plain, "attend": _attend_plain}[c["kind"]](st)
    if c["kind"] == "norm":
        codes, scales, values = _ctx().rmsnorm_quant(
            st["x"], residual=st["residual"], residual_out=st["sum"], gain=st["gain"], eps=1e-6, bits=c["bits"],
            clip=c["clip"], codes=st["codes"], scales=st["scales"], values=None if c["out"] == "codes" else st["values"])
        if c["out"] == "codes":  # what the codes stand for
            values = torch.mul(codes, scales[:, None], out=st["values"])
        return {"values": values, "scales": scales, "sum": st["sum"]}
    if c["kind"] == "append":
        _ctx().kv_append(st["cache"], st["batch"], st["q"], st["k"], st["v"], rope=st["rope"], hadamard=c["hadamard"],
                         asymmetric=c["asym"], clip=c["clip"], q_out=st["q_out"], k_values=st["k_values"],
                         v_values=st["v_values"])
        return {x: st[x] for x in ("q_out", "k_values", "v_values", "k_steps", "v_steps")}
    _ctx().kv_attend(st["cache"], st["batch"], st["q"], out=st["out"], lse=st["lse"], window=c["window"])
    return {"out": st["out"], "lse": st["lse"]}


# ------------------------------------------------------------------------------------- from the definition, in 64 bits
def _steps64(y, bits, clip, asym):
    """Values, steps and shifts in 64 bits.  Which code an entry gets is decided in float32, by definition: entries that are
    bfloat16 lie on the borders between two codes often, and there only the defined roundings tell."""
    clip = torch.tensor(clip, dtype=torch.float32, device=DEV)
    y32 = y.float()
    if asym:
        lo, hi = 0, 2**bits - 1
        low, high = clip * y32.min(-1, keepdim=True).values, clip * y32.max(-1, keepdim=True).values
        b = clip.double() * y.min(-1, keepdim=True).values
        s = (clip.double() * y.max(-1, keepdim=True).values - b) / hi
    else:
        hi = 2 ** (bits - 1) - 1
        lo = -hi
        low, high = 0.0, clip * y32.abs().max(-1, keepdim=True).values
        b = torch.zeros_like(y[..., :1])
        s = clip.double() * y.abs().max(-1, keepdim=True).values / hi
    step = torch.div(high - low, torch.tensor(float(hi), device=DEV))
    code = torch.clamp(torch.round(torch.div(y32 - low, step)), lo, hi).double()
    return torch.where(step > 0, code, 0.0) * s + b, s, b


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "norm":
        h = st["x"].double()
        total = None
        if st["residual"] is not None:
            total = h + st["residual"].double()
            h = total.to(st["x"].dtype).double()  # the norm is that of the stored sum
        y = h * (1.0 / torch.sqrt((h * h).sum(1, keepdim=True) / case["d"] + 1e-6)).float().double()  # a float32 factor
        if st["gain"] is not None:
            y = y * st["gain"].double()
        v, s, _ = _steps64(y, case["bits"], case["clip"], False)
        return {"values": v, "scales": s[:, 0], "sum": total}
    rows, lens = _sizes(case)
    hd, h, hq, page = case["head_dim"], case["heads"], case["q_heads"], case["page"]
    table = st["page_table"].cpu()
    if case["kind"] == "append":
        had = torch.ones(1, 1, dtype=torch.float64, device=DEV)
        while had.shape[0] < hd:
            had = torch.cat((torch.cat((had, had), 1), torch.cat((had, -had), 1)), 0)
        had = had / math.sqrt(hd)
        res = {x: st[x].double() for x in ("q_out", "k_values", "v_values", "k_steps", "v_steps")}
        at = 0
        for s, (r, n) in enumerate(zip(rows, lens)):
            pos = torch.arange(n - r, n, device=DEV)
            parts = {}
            for x in "qkv":
                y = st[x][at : at + r].double().reshape(r, -1, hd)
                if x != "v" and st["rope"] is not None:
                    t = st["rope"][pos].double()  # the table is an input
                    z = torch.complex(t[..., 0], t[..., 1])[:, None] * torch.complex(y[..., : hd // 2], y[..., hd // 2 :])
                    y = torch.cat((z.real, z.imag), -1)
                if x != "v" and case["hadamard"]:
                    y = y @ had
                parts[x] = y
            res["q_out"][at : at + r] = parts["q"].reshape(r, -1)
            where = table[s].to(DEV).long()[pos // page]
            for x in "kv":
                v, step, b = _steps64(parts[x], case["bits"], case["clip"], case["asym"])
                if not case["asym"]:  # held as codes from zero upwards: the shift is that of code zero
                    b = b - step * 2 ** (case["bits"] - 1)
                res[x + "_values"][at : at + r] = v.reshape(r, -1)
                for i in range(h):
                    res[x + "_steps"][where, i, pos % page] = torch.cat((step, b), -1)[:, i]
            at += r
        return res
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(out.shape[0], hq, dtype=torch.float64, device=DEV)
    at = 0
    for s, (r, n) in enumerate(zip(rows, lens)):
        pages = table[s, : -(-n // page)].to(DEV).long()
        held = {}
        for x in "kv":
            u = st[x + "_codes"][pages]
            if case["bits"] == 4:
                w = torch.empty(*u.shape[:-1], hd, dtype=torch.uint8, device=DEV)
                w[..., 0::2], w[..., 1::2] = u % 16, u // 16
                u = w
            d = st[x + "_steps"][pages].double()
            held[x] = (u.double() * d[..., 0, None] + d[..., 1, None]).permute(1, 0, 2, 3).reshape(h, -1, hd)[:, :n]
        pos = torch.arange(n - r, n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None]
        seen = (j <= pos) & ((j > pos - case["window"]) if case["window"] else True)
        for head in range(hq):
            q = st["q"][at : at + r, head * hd : (head + 1) * hd].double()
            a = q @ held["k"][head // (hq // h)].T / math.sqrt(hd)
            a = torch.where(seen, a, -math.inf)
            l = torch.logsumexp(a, 1)
            out[at : at + r, head * hd : (head + 1) * hd] = torch.exp(a - l[:, None]) @ held["v"][head // (hq // h)]
            lse[at : at + r, head] = l
        at += r
    return {"out": out, "lse": lse if case["lse"] else None}
