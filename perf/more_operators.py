"""Performance cases of the operators of a stage that is trained on packed documents with normed queries and keys, and that
keeps what backward-p2 needs in 8 bits.

Kinds of case:
  norm      norms of the query and key heads with the rotary positions in the same pass: "step" (forward, backward-p1 and the gains'
            gradient), "append" (new tokens: q normed and rotated, k into the cache, v into the cache)
  packed    causal attention over sequences of different lengths that lie one behind the other: "fwd", "step" (forward and
            backward-p1)
  stash     tensors kept in 8 bits with a scale for up to 1024 tokens of a column: "keep" (stored, and taken out again), "dw" (the
            inputs and output derivatives of a linear layer stored per micro-batch, and the weight gradient from them)

With own = False the operators are computed in plain torch operations in 32 bits; with own = True by this library.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
BLOCK = 1024                    # tokens of a column that share a scale


# ----------------------------------------------------------------------------------------------------------- cases
def _norm(name, op, batch, tokens, heads, kv_heads, head_dim, rot_dim, dtype, interleaved=False, positions=False, n_pos=0,
          capacity=0, sinks=0):
    """tokens: per sequence (append: new ones); positions: given per token rather than restarting in every sequence; n_pos: rows
    of the table; capacity, sinks: of the cache (append)."""
    return {"name": name, "kind": "norm", "op": op, "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rot_dim": rot_dim, "dtype": dtype, "interleaved": interleaved, "positions": positions,
            "n_pos": n_pos, "capacity": capacity, "sinks": sinks}


def _packed(name, op, rows, seqs, spread, heads, kv_heads, head_dim, behind=0):
    """seqs sequences in rows - behind rows, the longest `spread` times as long as the shortest; `behind`: rows of no sequence at
    the end."""
    return {"name": name, "kind": "packed", "op": op, "rows": rows, "seqs": seqs, "spread": spread, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "behind": behind}


def _stash(name, op, micro_batches, tokens, cols, other, dtype):
    """cols: of the tensor (dw: the layer's inputs); other: of its output derivatives (dw)."""
    return {"name": name, "kind": "stash", "op": op, "micro_batches": micro_batches, "tokens": tokens, "cols": cols, "other": other, "dtype": dtype}


def listed():
    return [
        # a layer of the 7B stage with grouped heads: forward and backward of a micro-batch of documents, whose positions are given
        _norm("norm_step_7b", "step", 2, 4096, 32, 8, 128, 128, "bf16", positions=True, n_pos=4096),
        # a small fp32 model on sequences of odd length, a third of a head's columns rotated in interleaved pairs
        _norm("norm_step_odd", "step", 3, 333, 6, 2, 96, 32, "f32", interleaved=True, n_pos=333),
        # the next token of some answers, into ring caches: latency counts
        _norm("norm_append", "append", 16, 1, 32, 8, 128, 128, "bf16", n_pos=16384, capacity=1028, sinks=4),
        # prompts of very different lengths, answered together
        _packed("packed_fwd_prompts", "fwd", 8192, 24, 40, 32, 8, 128),
        # the training step of a layer on documents packed to twice the stage's longest sequence: the largest call
        _packed("packed_step_docs", "step", 8192, 5, 12, 32, 8, 128),
        # a small model on many short documents, with rows to spare
        _packed("packed_step_short", "step", 4096, 61, 30, 12, 4, 64, behind=77),
        # one short prompt: latency counts
        _packed("packed_fwd_one", "fwd", 200, 1, 1, 32, 8, 128),
        # a micro-batch's SwiGLU output of the 7B stage, kept and taken out again
        _stash("stash_keep_7b", "keep", 1, 4096, 11008, 0, "bf16"),
        # the smallest: the fp32 benchmark stage's, where latency counts
        _stash("stash_keep_tiny", "keep", 1, 129, 256, 0, "f32"),
        # the 7B stage's down projection over a whole step
        _stash("stash_dw_7b", "dw", 8, 4096, 11008, 4096, "bf16"),
        # its output projection at the shorter context, one micro-batch after the other
        _stash("stash_dw_s1024", "dw", 4, 1024, 4096, 4096, "bf16"),
        # odd sizes: tokens and columns that end inside a tile
        _stash("stash_dw_odd", "dw", 3, 333, 520, 1001, "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    kind = rng.choice(["norm", "packed", "stash"])
    if kind == "norm":
        kv = rng.choice([1, 2, 4, 5, 8])
        heads = kv * rng.choice([1, 2, 3, 4, 8])
        dh = rng.choice([64, 96, 128, 128, 256])
        rot = rng.choice([dh, dh, dh // 2, 32])
        inter = rng.random() < 0.5
        if rng.random() < 0.35:
            sinks = rng.choice([0, 4, 17])
            return _norm("", "append", _log_int(rng, 1, 64), _log_int(rng, 1, 200), heads, kv, dh, rot, rng.choice(["bf16", "bf16", "f32"]), inter,
                         n_pos=_log_int(rng, 1000, 100000), capacity=sinks + _log_int(rng, 16, 2000), sinks=sinks)
        tokens, positions = _log_int(rng, 1, 4096), rng.random() < 0.5
        return _norm("", "step", rng.choice([1, 1, 2, 3, 4]), tokens, heads, kv, dh, rot, rng.choice(["bf16", "bf16", "f32"]), inter, positions,
                     max(tokens, _log_int(rng, 1000, 100000)) if positions else tokens)
    if kind == "packed":
        kv = rng.choice([1, 2, 4, 5, 8])
        heads = kv * rng.choice([1, 2, 3, 4, 5, 8])
        rows = _log_int(rng, 1, 8192)
        behind = rng.randrange(rows) if rng.random() < 0.2 else 0
        seqs = min(_log_int(rng, 1, 100), rows - behind)
        return _packed("", rng.choice(["fwd", "step"]), rows, seqs, rng.choice([1, 4, 30]), heads, kv, rng.choice([64, 128]), behind)
    if rng.random() < 0.4:
        return _stash("", "keep", 1, _log_int(rng, 1, 8192), _log_int(rng, 16, 12288), 0, rng.choice(["bf16", "bf16", "f32"]))
    return _stash("", "dw", rng.choice([1, 2, 3, 4, 8]), _log_int(rng, 32, 4096), _log_int(rng, 64, 11008), _log_int(rng, 64, 11008),
                  rng.choice(["bf16", "bf16", "f32"]))


def draw(rng):
    largest = {}
    for c in listed():
        w, have = work(c), largest.setdefault(c["kind"], {"bytes": 0, "flops": 0})
        for k in have:
            have[k] = max(have[k], w[k])
    while True:
        case = _draw_one(rng)
        w, most = work(case), largest[case["kind"]]
        # (the plain form of the attention pads every sequence to the longest)
        padded = case["seqs"] * case["heads"] * max(_lengths(case)) ** 2 if case["kind"] == "packed" else 0
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and padded <= 5 * 32 * 4096 ** 2:
            del case["name"]
            return case


# ---------------------------------------------------------------------------------------------------------- inputs
def _tdtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def _append_lengths(case):
    """Tokens of every sequence after the new ones: spread over the table's positions, the shortest with no history."""
    B, n, top = case["batch"], case["tokens"], case["n_pos"]
    return [n + ((top - n) * b) // B if top > n else n for b in range(B)]


def _lengths(case):
    """Tokens of every sequence: a geometric spread, in no order."""
    n, used = case["seqs"], case["rows"] - case["behind"]
    weight = [case["spread"] ** (((5 * b + 2) % n) / n) for b in range(n)]
    left, out = used, []
    for b in range(n):
        share = int(round(left * weight[b] / sum(weight[b:])))
        out.append(left if b == n - 1 else max(1, min(share, left - (n - 1 - b))))
        left -= out[-1]
    return out


def _angles64(case):
    r = case["rot_dim"]
    theta = 10000.0 ** (-torch.arange(r // 2, dtype=torch.float64, device=DEV) * 2 / r)
    return torch.arange(case["n_pos"], dtype=torch.float64, device=DEV)[:, None] * theta


def _norm_inputs(case, seed):
    """Heads behind a projection, of a scale that differs from column to column; gains near 1; derivatives ~ N(0, 1)."""
    g, B, n, dt, dh = _generator(seed), case["batch"], case["tokens"], _tdtype(case["dtype"]), case["head_dim"]
    qk, kvw = (case["heads"] + case["kv_heads"]) * dh, case["kv_heads"] * dh
    ang = _angles64(case)
    scale = torch.exp(0.5 * torch.randn((qk + kvw,), generator=g, device=DEV))
    s = {"table": torch.stack([torch.cos(ang), torch.sin(ang)], dim=-1).float().contiguous(),
         "gq": (1 + 0.1 * torch.randn((dh,), generator=g, device=DEV)).to(dt), "gk": (1 + 0.1 * torch.randn((dh,), generator=g, device=DEV)).to(dt),
         "qkv": (torch.randn((B * n, qk + kvw), generator=g, device=DEV) * scale).to(dt)}
    if case["op"] == "append":
        shape = (B, case["capacity"], kvw)
        s["cache_k"], s["cache_v"] = _normal(g, shape, dt), _normal(g, shape, dt)
        s["lengths"] = torch.tensor(_append_lengths(case), dtype=torch.int32, device=DEV)
    else:
        s["d_qk"] = _normal(g, (B * n, qk), dt)
        s["positions"] = torch.randint(0, case["n_pos"], (B * n,), generator=g, device=DEV, dtype=torch.int32) if case["positions"] else None
    return s


def _packed_inputs(case, seed):
    """Heads and derivatives ~ N(0, 1) (rotated heads have that scale behind a norm)."""
    g, dh = _generator(seed), case["head_dim"]
    qw, kvw = case["heads"] * dh, case["kv_heads"] * dh
    s = {"qkv": _normal(g, (case["rows"], qw + 2 * kvw), torch.bfloat16)}
    if case["op"] == "step":
        s["d_out"] = _normal(g, (case["rows"], qw), torch.bfloat16)
    return s


def _stash_inputs(case, seed):
    """Activations of scales that differ from column to column, and derivatives, small, with one token in eight left out of the loss."""
    g, dt, shape = _generator(seed), _tdtype(case["dtype"]), (case["micro_batches"], case["tokens"], case["cols"])
    s = {"x": (torch.randn(shape, generator=g, device=DEV) * torch.exp(torch.randn((case["cols"],), generator=g, device=DEV))).to(dt)}
    if case["op"] == "dw":
        dy = torch.randn((*shape[:2], case["other"]), generator=g, device=DEV).mul_(1e-4)
        dy *= torch.rand((*shape[:2], 1), generator=g, device=DEV) >= 0.125
        s["dy"] = dy.to(dt)
    return s


def prepare(case, seed):
    state = {"case": case}
    if case["kind"] == "norm":
        state.update(_norm_inputs(case, seed))
    elif case["kind"] == "packed":
        n = _lengths(case)
        state.update(_packed_inputs(case, seed))
        state["starts"] = torch.tensor([sum(n[:b]) for b in range(len(n) + 1)], dtype=torch.int32, device=DEV)
        state["longest"] = max(n)
    else:
        state.update(_stash_inputs(case, seed))
    if own:
        import paper_2405_18047_amd as tbp
        state["tbp"] = tbp
        if case["kind"] == "stash":
            # the stash of a stage, which lives from step to step
            state["kept"] = tbp.Stash8(case["tokens"], case["cols"], case["micro_batches"], state["x"].dtype, device=DEV)
            if case["op"] == "dw":
                state["d_kept"] = tbp.Stash8(case["tokens"], case["other"], case["micro_batches"], state["x"].dtype, device=DEV)
    return state


# ------------------------------------------------------------------------------------------------- the framework's
def _run_own(state):
    case, tbp = state["case"], state["tbp"]
    if case["kind"] == "norm":
        heads = (state["gq"], state["gk"], case["heads"], case["kv_heads"], case["head_dim"], EPS, state["table"])
        layout = tbp.TBP_ROTARY_INTERLEAVED if case["interleaved"] else tbp.TBP_ROTARY_HALF
        if case["op"] == "append":
            q = tbp.tbp_qk_norm_append(state["qkv"], *heads, state["lengths"], state["cache_k"], state["cache_v"], sinks=case["sinks"], layout=layout)
            return q, state["cache_k"], state["cache_v"]
        where = {"positions": state["positions"], "seq": case["tokens"], "layout": layout}
        y = tbp.tbp_qk_norm(state["qkv"], *heads, **where)
        dx, parts = tbp.tbp_qk_norm_p1(state["d_qk"], state["qkv"], *heads, **where)
        return y, dx, tbp.tbp_gain_partials_sum(parts)
    if case["kind"] == "packed":
        heads = (case["heads"], case["kv_heads"], case["head_dim"])
        out, lse = tbp.tbp_packed_attention_fwd(state["qkv"], state["starts"], *heads)
        if case["op"] == "fwd":
            return out, lse
        return out, lse, tbp.tbp_packed_attention_p1(state["qkv"], out, state["d_out"], lse, state["starts"], *heads)
    kept = state["kept"]
    if case["op"] == "keep":
        kept.put(0, state["x"][0])
        return kept.get(0)
    for mb in range(case["micro_batches"]):
        kept.put(mb, state["x"][mb])
        state["d_kept"].put(mb, state["dy"][mb])
    return tbp.tbp_stash8_dw(kept, state["d_kept"])


# --------------------------------------------------------------------------------------------------- the plain form
def _rotate(x, cs, interleaved, sign):
    """x [rows, heads, dh] in 32 bits; cs [rows, r / 2, 2]."""
    half = cs.shape[1]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * sign
    ya, yb = a * c - b * s, a * s + b * c
    y = torch.stack([ya, yb], dim=-1).flatten(-2) if interleaved else torch.cat([ya, yb], dim=-1)
    return torch.cat([y, rest], dim=-1)


def _plain_norm(state):
    case, qkv = state["case"], state["qkv"]
    B, n, H, KV, dh, inter = (case[k] for k in ("batch", "tokens", "heads", "kv_heads", "head_dim", "interleaved"))
    rows, qk, dt = B * n, (H + KV) * dh, qkv.dtype
    x = qkv[:, :qk].float().view(rows, H + KV, dh)
    gain = torch.cat([state["gq"].float().expand(H, dh), state["gk"].float().expand(KV, dh)])
    inv = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
    normed = x * inv
    if case["op"] == "step":
        pos = state["positions"].long() if state["positions"] is not None else torch.arange(rows, device=DEV) % n
        cs = state["table"][pos]
        y = _rotate(normed * gain, cs, inter, 1.0).reshape(rows, qk).to(dt)
        dz = _rotate(state["d_qk"].float().view(rows, H + KV, dh), cs, inter, -1.0)
        dn = dz * gain
        dx = inv * (dn - normed * (dn * normed).mean(dim=-1, keepdim=True))
        dg = (dz * normed).sum(dim=0, dtype=torch.float64)
        dg = torch.stack([dg[:H].sum(dim=0), dg[H:].sum(dim=0)]).float()
        return y, dx.reshape(rows, qk).to(dt), dg.reshape(2 * dh)
    sinks, ring = case["sinks"], case["capacity"] - case["sinks"]
    pos = (state["lengths"].long()[:, None] - n + torch.arange(n, device=DEV)).reshape(-1)
    known = (pos < case["n_pos"])[:, None, None]
    y = torch.where(known, _rotate(normed * gain, state["table"][pos.clamp(max=case["n_pos"] - 1)], inter, 1.0), math.nan).reshape(rows, qk).to(dt)
    seq = torch.arange(B, device=DEV).repeat_interleave(n)
    slot = torch.where(pos < sinks, pos, sinks + torch.remainder(pos - sinks, ring))
    stays = (pos < sinks) | (pos >= state["lengths"].long()[seq] - ring)      # not taken over by a later one of these tokens
    seq, slot = seq[stays], slot[stays]
    state["cache_k"][seq, slot] = y[stays][:, H * dh:]
    state["cache_v"][seq, slot] = qkv[stays][:, qk:]
    return y[:, :H * dh].contiguous(), state["cache_k"], state["cache_v"]


def _plain_packed(state):
    """Every sequence padded to the longest, the query heads of a key head one below the other."""
    case, qkv, n = state["case"], state["qkv"], state["longest"]
    B, H, KV, dh, rows = (case[k] for k in ("seqs", "heads", "kv_heads", "head_dim", "rows"))
    starts, scale, G = state["starts"].long(), 1.0 / math.sqrt(dh), H // KV
    i = torch.arange(n, device=DEV)
    there = i < (starts[1:] - starts[:-1])[:, None]                           # [B, n]
    at = torch.where(there, starts[:-1, None] + i, 0)

    def spread(t, heads):
        """[rows, KV heads dh] -> [B, KV, heads n, dh]"""
        return torch.where(there[..., None], t[at].float(), 0.0).view(B, n, KV, heads, dh).permute(0, 2, 3, 1, 4).reshape(B, KV, heads * n, dh)

    def gather(t, heads):
        t = t.reshape(B, KV, heads, n, dh).permute(0, 3, 1, 2, 4).reshape(B, n, KV * heads * dh)
        out = torch.zeros((rows, KV * heads * dh), dtype=qkv.dtype, device=DEV)
        out[at[there]] = t[there].to(qkv.dtype)
        return out

    q, k, v = spread(qkv[:, :H * dh], G), spread(qkv[:, H * dh:(H + KV) * dh], 1), spread(qkv[:, (H + KV) * dh:], 1)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(B, KV, G, n, n)
    s.masked_fill_(i[None, :] > i[:, None], -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    lse = torch.full((H, rows), -math.inf, device=DEV)
    lse[:, at[there]] = ((m + torch.log(l)) / math.log(2.0)).reshape(B, H, n).permute(1, 0, 2)[:, there]
    p = p.div_(l).view(B, KV, G * n, n)
    o = torch.matmul(p, v)
    out = gather(o, G)
    if case["op"] == "fwd":
        return out, lse
    do = spread(state["d_out"], G)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(dim=-1, keepdim=True)).mul_(p)
    dq, dk = torch.matmul(ds, k).mul_(scale), torch.matmul(ds.transpose(2, 3).contiguous(), q).mul_(scale)
    return out, lse, torch.cat([gather(dq, G), gather(dk, 1), gather(dv, 1)], dim=1)


def _power(e):
    """2^e in 32 bits, exactly (e in -126 .. 127)."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _held(x):
    """The values that x [micro-batches, tokens, columns] is held as, in 32 bits: of every 1024 tokens of a column (from the first token of the
    micro-batch on) whole multiples, -127 .. 127, of the smallest power of two with which the largest one is in that range."""
    M, n, c = x.shape
    tall = min(n, BLOCK)
    b = torch.cat([x.float(), torch.zeros((M, -n % tall, c), device=DEV)], dim=1).view(M, -1, tall, c)
    part, exponent = torch.frexp(b.abs().amax(dim=2, keepdim=True))           # part in 1/2 .. 1
    e = (exponent - 7 + (part > 127 / 128).int()).clamp(min=-126)
    return (torch.round(b * _power(-e)) * _power(e)).view(M, -1, c)[:, :n]


def _plain_stash(state):
    case, x = state["case"], state["x"]
    held = _held(x)
    if case["op"] == "keep":
        return held[0].to(x.dtype)
    return torch.matmul(held.reshape(-1, case["cols"]).t(), _held(state["dy"]).reshape(-1, case["other"]))


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "packed": _plain_packed, "stash": _plain_stash}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------------------ work
def work(case):
    """Every input read once, every output written once; of the attention's products the pairs that are seen."""
    e = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if case["kind"] == "norm":
        rows, dh = case["batch"] * case["tokens"], case["head_dim"]
        qk = rows * (case["heads"] + case["kv_heads"]) * dh
        if case["op"] == "append":
            return {"bytes": 2 * e * (qk + rows * case["kv_heads"] * dh) + 4 * rows * case["rot_dim"], "flops": 7 * qk}
        table = 4 * case["rot_dim"] * min(rows, case["n_pos"])
        return {"bytes": 4 * e * qk + table + 8 * dh, "flops": 18 * qk}
    if case["kind"] == "packed":
        H, KV, dh, rows = (case[k] for k in ("heads", "kv_heads", "head_dim", "rows"))
        pairs = sum(n * (n + 1) // 2 for n in _lengths(case)) * H
        qkv = (H + 2 * KV) * dh
        nbytes = rows * (2 * qkv + 2 * H * dh + 4 * H)
        if case["op"] == "fwd":
            return {"bytes": nbytes, "flops": 4 * dh * pairs}
        return {"bytes": nbytes + rows * (2 * H * dh + 2 * qkv), "flops": 14 * dh * pairs}
    rows = case["micro_batches"] * case["tokens"]
    if case["op"] == "keep":
        return {"bytes": 2 * e * rows * case["cols"], "flops": 4 * rows * case["cols"]}
    return {"bytes": e * rows * (case["cols"] + case["other"]) + 4 * case["cols"] * case["other"], "flops": 2 * rows * case["cols"] * case["other"]}


# ----------------------------------------------------------------------------------------------------------- exact
def _turn(x, ang, interleaved, back):
    """x [rows, heads, dh]: the pairs as complex numbers, times exp(i angle)."""
    half, x = ang.shape[1], x.clone()
    at = [torch.arange(half, device=DEV) * 2 + o if interleaved else torch.arange(half, device=DEV) + o * half for o in (0, 1)]
    z = torch.complex(x[:, :, at[0]], x[:, :, at[1]]) * torch.polar(torch.ones_like(ang), -ang if back else ang)[:, None]
    x[:, :, at[0]], x[:, :, at[1]] = z.real, z.imag
    return x


def _exact_norm(case, seed):
    s = _norm_inputs(case, seed)
    B, n, H, KV, dh, inter = (case[k] for k in ("batch", "tokens", "heads", "kv_heads", "head_dim", "interleaved"))
    qk, ang = (H + KV) * dh, _angles64(case)

    def forward(x, gq, gk):
        g = torch.cat([gq.expand(H, dh), gk.expand(KV, dh)])
        return x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * g

    if case["op"] == "step":
        ang = ang[s["positions"].long()] if case["positions"] else ang[:n].repeat(B, 1)
        y, dx, dg = [], [], torch.zeros((2, dh), dtype=torch.float64, device=DEV)
        for r in range(0, B * n, 1024):
            rows = slice(r, min(r + 1024, B * n))
            x = s["qkv"][rows, :qk].double().view(-1, H + KV, dh).requires_grad_()
            g = [s[k].double().requires_grad_() for k in ("gq", "gk")]
            z = forward(x, *g)
            z.backward(_turn(s["d_qk"][rows].double().view(-1, H + KV, dh), ang[rows], inter, True))
            y.append(_turn(z.detach(), ang[rows], inter, False).reshape(-1, qk))
            dx.append(x.grad.reshape(-1, qk))
            dg += torch.stack([t.grad for t in g])
        return torch.cat(y), torch.cat(dx), dg.reshape(2 * dh)
    ck, cv, q = s["cache_k"].double(), s["cache_v"].double(), []
    for b, length in enumerate(_append_lengths(case)):
        rows = slice(b * n, (b + 1) * n)
        at = torch.arange(length - n, length, device=DEV)
        z = forward(s["qkv"][rows, :qk].double().view(n, H + KV, dh), s["gq"].double(), s["gk"].double())
        y = _turn(z, ang[at.clamp(max=case["n_pos"] - 1)], inter, False)
        y = torch.where((at < case["n_pos"])[:, None, None], y, math.nan).reshape(n, qk)
        q.append(y[:, :H * dh])
        for i in range(n):                                       # in order: a later token takes an earlier one's slot over
            p = length - n + i
            slot = p if p < case["sinks"] else case["sinks"] + (p - case["sinks"]) % (case["capacity"] - case["sinks"])
            ck[b, slot], cv[b, slot] = y[i, H * dh:], s["qkv"][b * n + i, qk:].double()
    return torch.cat(q), ck, cv


def _exact_packed(case, seed):
    s = _packed_inputs(case, seed)
    H, KV, dh, rows = (case[k] for k in ("heads", "kv_heads", "head_dim", "rows"))
    G, step, first = H // KV, case["op"] == "step", 0
    out = torch.zeros((rows, H * dh), dtype=torch.float64, device=DEV)
    lse = torch.full((H, rows), -math.inf, dtype=torch.float64, device=DEV)
    dqkv = torch.zeros_like(s["qkv"], dtype=torch.float64)
    for m in _lengths(case):                                     # one sequence and one head at a time
        hidden = torch.ones((m, m), dtype=torch.bool, device=DEV).triu(1)
        at = slice(first, first + m)
        first += m
        for h in range(H):
            cols = [slice((x + y) * dh, (x + y + 1) * dh) for x, y in ((0, h), (H, h // G), (H + KV, h // G))]
            q, k, v = (s["qkv"][at, c].double().requires_grad_(step) for c in cols)
            scores = (q @ k.t() / math.sqrt(dh)).masked_fill(hidden, -math.inf)
            o = torch.softmax(scores, dim=1) @ v
            out[at, cols[0]] = o.detach()
            lse[h, at] = torch.logsumexp(scores.detach(), dim=1) / math.log(2.0)
            if step:
                o.backward(s["d_out"][at, cols[0]].double())
                for c, t in zip(cols, (q, k, v)):
                    dqkv[at, c] += t.grad
    return (out, lse, dqkv) if step else (out, lse)


def _nearest(x):
    """The definition: the nearest multiple of the scale, halves to the even one."""
    M, n, c = x.shape
    held = torch.empty((M, n, c), dtype=torch.float64, device=DEV)
    for t in range(0, n, BLOCK):
        b = x[:, t:t + BLOCK].double()
        part, e = torch.frexp(b.abs().amax(dim=1, keepdim=True) / 127)
        e = torch.where(part == 0.5, e - 1, e).clamp(min=-126)                # the power of two at or above the quotient
        scale = ((e.long() + 1023) << 52).view(torch.float64)
        a = b.abs() / scale
        whole = torch.floor(a)
        up = (a - whole > 0.5) | ((a - whole == 0.5) & (torch.remainder(whole, 2) == 1))
        held[:, t:t + BLOCK] = (whole + up) * scale * torch.sign(b)
    return held


def _exact_stash(case, seed):
    s = _stash_inputs(case, seed)
    if case["op"] == "keep":
        return _nearest(s["x"])[0]
    dw = torch.zeros((case["cols"], case["other"]), dtype=torch.float64, device=DEV)
    for mb in range(case["micro_batches"]):
        dw += _nearest(s["x"][mb:mb + 1])[0].t() @ _nearest(s["dy"][mb:mb + 1])[0]
    return dw


def exact(case, seed):
    return {"norm": _exact_norm, "packed": _exact_packed, "stash": _exact_stash}[case["kind"]](case, seed)
