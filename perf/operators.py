"""The store's operators beyond the gate: rotary positions with the append, the cache held in 4 bits, attention over it.

Three kinds of case:
  rope  rotary positions on several axes turned into q and k while k and v go into the cache's pages (append_rope)
  pack  completed chunks of the cache to 4 bits, and the values they stand for (pack_chunks, unpack_chunks)
  attn  decode attention over [chunks held in 4 bits ; recent rows in bf16] (decode_attn_q4)

4 bits: each row (one token's key or value in one head, 128 numbers) has two groups of 64.  A group keeps its smallest value `low`, a
scale = bf16((largest - smallest) / 15) and a code 0..15 per number: how many of the borders low + (k + 1/2) scale, k = 0..14, lie below
it (a number on a border takes the lower code).  It stands for low + code * scale.
"""
import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
DEV = "cuda"


# ---- the cases ----------------------------------------------------------------------------------------------------------------------

def _rope(name, **kw):
    # n0: tokens stored before; n: new ones; axes: 1 (text) or 3 (time, height, width); fused: q, k, v are views of one projection's output
    c = dict(name=name, kind="rope", B=1, Hq=8, Hkv=8, n0=0, n=1, axes=1, adjacent=False, fused=True, far=0, C=64)
    return {**c, **kw}


def _pack(name, **kw):
    # chunks [first, first + chunks) of every sequence
    return {**dict(name=name, kind="pack", B=1, H=8, C=64, first=0, chunks=1), **kw}


def _attn(name, **kw):
    # T query tokens on Hq heads, Hq / Hkv of which share a key head; gated: only the chunks of the keep list, about `keep` of them
    return {**dict(name=name, kind="attn", B=1, Hq=8, Hkv=8, n=2048, C=64, W=256, T=1, causal=False, gated=False, keep=0.5), **kw}


def listed():
    return [
        # one decoded token of one robot: latency alone
        _rope("rope_token_b1_h8", n0=2047),
        # seven action tokens of a batch, 32 query heads on 8 key heads, far into a long episode
        _rope("rope_actions_b16_q32_kv8", B=16, Hq=32, Hkv=8, n0=16505, n=7, far=1000000),
        # a camera frame of 250 patches: height and width beside the time of the frame
        _rope("rope_frame_b3_h20", B=3, Hq=20, Hkv=20, n0=500, n=250, axes=3, fused=False),
        # a long prompt of video and text, adjacent pairs
        _rope("rope_prompt_b8_h32_n4096", B=8, Hq=32, Hkv=32, n=4096, axes=3, adjacent=True),
        # the trigger: one chunk of every sequence has left the window
        _pack("pack_chunk_b4_h32_c64", B=4, H=32, first=59),
        # a whole prefilled cache
        _pack("pack_b8_h32_n3584", B=8, H=32, chunks=56),
        # one robot, short history: latency alone
        _attn("attn_b1_h8_n2048"),
        # the paper's path at its usual size: gated history, odd tail
        _attn("attn_b4_h32_n4167_gated", B=4, Hq=32, Hkv=32, n=4167, gated=True),
        # grouped heads, one token
        _attn("attn_b8_q32_kv8_n4099", B=8, Hq=32, Hkv=8, n=4099, W=512),
        # seven action tokens decoded together, causal
        _attn("attn_actions_b16_q32_kv8_n16512", B=16, Hq=32, Hkv=8, n=16512, C=128, W=1024, T=7, causal=True),
        # one very long history: the work is split along it
        _attn("attn_b1_q32_kv8_n100003", Hq=32, n=100003),
        # the largest: full batch, long gated history
        _attn("attn_b16_h32_n16512_gated", B=16, Hq=32, Hkv=32, n=16512, C=128, W=1024, gated=True),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    kind = rng.choice(["rope", "pack", "attn"])
    Hkv = rng.choice([1, 2, 4, 5, 8, 20, 32])
    if kind == "rope":
        B, G = _log(rng, 1, 16), rng.choice([1, 1, 2, 4, 7])
        n = _log(rng, 1, max(1, min(4096, 8 * 32 * 3 * 4096 // (B * Hkv * (G + 2)))))
        return _rope("", B=B, Hkv=Hkv, Hq=Hkv * G, n=n, n0=rng.choice([0, _log(rng, 1, 5000)]), axes=rng.choice([1, 2, 3]), adjacent=rng.random() < 0.5,
                     fused=rng.random() < 0.6, far=rng.choice([0, _log(rng, 1, 10000000)]), C=rng.choice([16, 24, 32, 64, 100, 128]))
    C = rng.choice([16, 32, 48, 64, 128, 256])
    if kind == "pack":
        B = _log(rng, 1, 16)
        chunks = _log(rng, 1, max(1, min(4096 // C, 8 * 32 * 3584 // (B * Hkv * C))))
        return _pack("", B=B, H=Hkv, C=C, first=_log(rng, 1, 20) - 1, chunks=chunks)
    B, G = _log(rng, 1, 16), rng.choice([1, 1, 2, 4, 7, 8])
    T = rng.choice([1, 1, 1, 2, 5, 7, 16])
    n = _log(rng, 1, max(1, min(60000, 16 * 32 * 16512 // (B * Hkv))))
    return _attn("", B=B, Hkv=Hkv, Hq=Hkv * G, n=max(n, T), C=C, W=max(T, rng.choice([16, 100, 256, 1024])), T=T, causal=rng.random() < 0.5,
                 gated=rng.random() < 0.5, keep=rng.choice([0.1, 0.5, 0.9, 1.0]))


def _stale(c):
    return max(0, c["n"] - c["W"]) // c["C"]


def work(case):
    c = case
    if c["kind"] == "rope":
        rows = c["B"] * c["n"] * (c["Hq"] + 2 * c["Hkv"])
        return {"bytes": rows * 2 * 2 * D + 4 * c["B"] * c["n"] * c["axes"], "flops": 3 * D * c["B"] * c["n"] * (c["Hq"] + c["Hkv"])}
    if c["kind"] == "pack":
        rows = 2 * c["B"] * c["H"] * c["C"] * c["chunks"]      # keys and values; bf16 rows in, 72 bytes of codes and scales out, the values out
        return {"bytes": rows * (2 * D + 72 + 2 * D), "flops": rows * D * 6}
    nc = _stale(c)
    rows4 = nc * c["C"] * (c["keep"] if c["gated"] else 1.0)
    rows16 = c["n"] - nc * c["C"]
    S, queries = c["B"] * c["Hkv"], c["B"] * c["T"] * c["Hq"]
    return {"bytes": S * (rows4 * 2 * 72 + rows16 * 2 * 2 * D) + queries * (2 * 2 * D + 4), "flops": 4 * D * queries * (rows4 + rows16)}


# ---- inputs -------------------------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _rope_inputs(c, seed):
    """q, k, v [B, n, heads, 128] bf16, positions [B, n, axes] int32"""
    g = _generator(seed)
    B, n = c["B"], c["n"]
    heads = [c["Hq"], c["Hkv"], c["Hkv"]]
    if c["fused"]:
        q, k, v = _normal(g, B, n, sum(heads), D).split(heads, dim=2)
    else:
        q, k, v = (_normal(g, B, n, h, D) for h in heads)
    i = torch.arange(n, device=DEV)
    width = max(1, math.isqrt(n))
    start = torch.randint(0, c["far"] + 1, (B, 1), generator=g, device=DEV)
    time = start + c["n0"] + (i if c["axes"] == 1 else i // 250)
    axes = [time, (i // width).expand(B, n), (i % width).expand(B, n)][:c["axes"]]
    return q, k, v, torch.stack(axes, dim=-1).to(torch.int32).contiguous()


def _frequencies(axes):
    """radians per position of the 64 pairs, and the axis each of them follows"""
    sections = {1: [64], 2: [40, 24], 3: [16, 24, 24]}[axes]
    return [10000.0 ** (-2.0 * j / D) for j in range(D // 2)], sum(([a] * s for a, s in enumerate(sections)), []), sections


def _cache_inputs(c, seed, S, n, C):
    """k, v [S, n, 128] bf16: unit normal, the keys with an offset of their own in every chunk"""
    g = _generator(seed)
    chunks = -(-n // C)
    offset = 0.5 * torch.randn(S, chunks, 1, D, generator=g, device=DEV)
    k = torch.randn(S, chunks, C, D, generator=g, device=DEV).add_(offset).to(torch.bfloat16).reshape(S, chunks * C, D)[:, :n].contiguous()
    return k, _normal(g, S, n, D), g


def _attn_inputs(c, seed):
    S, nc = c["B"] * c["Hkv"], _stale(c)
    k, v, g = _cache_inputs(c, seed, S, c["n"], c["C"])
    q = _normal(g, c["B"], c["T"], c["Hq"], D)
    scores = torch.rand(S, max(nc, 1), generator=g, device=DEV)[:, :nc]
    return k, v, q, scores, 1.0 - c["keep"]


def _to4(x):
    """[..., rows, 128] bf16 -> codes, two of them to a byte, and the groups' scales and lowest values"""
    x = x.unflatten(-1, (2, 64)).double()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = (high - low) / 15.0
    step = torch.exp2(torch.frexp(scale).exponent.clamp(min=-125).double() - 8.0)
    scale = torch.round(scale / step) * step      # to the 8 bits of bf16
    code = torch.where(scale > 0, torch.ceil((x - low) / scale - 0.5), 0.0).clamp(0, 15).to(torch.uint8).flatten(-2)
    return code[..., 0::2] + code[..., 1::2] * 16, scale.squeeze(-1).to(torch.bfloat16), low.squeeze(-1).to(torch.bfloat16)


def _from4(codes, scale, low):
    """the values in 32 bits"""
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).unflatten(-1, (2, 64))
    return (code.float() * scale.unsqueeze(-1).float() + low.unsqueeze(-1).float()).flatten(-2)


def prepare(case, seed):
    c = case
    if own:
        from paper_2509_21354_b200 import binding as b
    if c["kind"] == "rope":
        q, k, v, positions = _rope_inputs(c, seed)
        state = dict(c=c, q=q, k=k, v=v, positions=positions)
        frequencies, axis, sections = _frequencies(c["axes"])
        total = c["n0"] + c["n"]
        capacity = -(-total // c["C"]) * c["C"]
        if own:
            state["rope"] = b.Rope(sections, theta=10000.0, layout="adjacent" if c["adjacent"] else "halves")
            st = state["store"] = b.Store(B=c["B"], H=c["Hkv"], C_=c["C"], W=c["C"], max_tokens=total, d_g=64, Hq=c["Hq"])
            state["cache"] = [p.view(c["B"] * c["Hkv"], capacity, D)[:, c["n0"]:total] for p in (st.k_pages, st.v_pages)]
            state["out"] = torch.empty(c["B"], c["n"], c["Hq"], D, dtype=torch.bfloat16, device=DEV)
        else:
            state["cache"] = [torch.zeros(c["B"] * c["Hkv"], capacity, D, dtype=torch.bfloat16, device=DEV)[:, c["n0"]:total] for _ in range(2)]
            state["frequencies"] = torch.tensor(frequencies, dtype=torch.float64, device=DEV)
            state["axis"] = torch.tensor(axis, device=DEV)
        return state
    if c["kind"] == "pack":
        S, n = c["B"] * c["H"], (c["first"] + c["chunks"]) * c["C"]
        k, v, _ = _cache_inputs(c, seed, S, n, c["C"])
        state = dict(c=c, k=k, v=v, rows=slice(c["first"] * c["C"], n))
        if own:
            st = state["store"] = b.Store(B=c["B"], H=c["H"], C_=c["C"], W=0, max_tokens=n, d_g=64)
            st.attach_q4()
            st.append(0, k, v)
            st.pack_chunks(0, 0, c["first"])
        return state
    k, v, q, scores, tau = _attn_inputs(c, seed)
    nc = _stale(c)
    split = nc * c["C"]
    state = dict(c=c, q=q, split=split)
    if own:
        st = state["store"] = b.Store(B=c["B"], H=c["Hkv"], C_=c["C"], W=c["W"], max_tokens=c["n"], d_g=64, Hq=c["Hq"], attend="raw")
        st.attach_q4(max_query_tokens=c["T"])
        st.append(0, k, v)
        if c["gated"] and nc:
            g = torch.Generator().manual_seed(seed)
            weight = lambda *shape: (torch.randn(*shape, generator=g) / 16).numpy()
            lstm = b.LstmWeights(dict(W_ih=weight(256, 256), W_hh=weight(256, 64), b_ih=weight(256), b_hh=weight(256), w_s=weight(64), b_s=0.0))
            st.refresh(0, None, lstm, tau)
            st.scores[0, :, :nc] = scores
            st.compact(0, tau)
        st.pack_chunks(0, 0, nc)
    else:
        state["k4"], state["v4"] = _to4(k[:, :split]), _to4(v[:, :split])
        state["k16"], state["v16"] = k[:, split:].contiguous(), v[:, split:].contiguous()
        state["scores"], state["tau"] = scores, tau
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------------------------

def _turn(x, angle, adjacent):
    """x [B, n, heads, 128], angle [B, n, 64] in 64 bits; the turning in 32"""
    x = x.float()
    cos, sin = torch.cos(angle).float().unsqueeze(2), torch.sin(angle).float().unsqueeze(2)
    a, b = (x[..., 0::2], x[..., 1::2]) if adjacent else (x[..., :64], x[..., 64:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return (torch.stack([a, b], dim=-1).flatten(-2) if adjacent else torch.cat([a, b], dim=-1)).to(torch.bfloat16)


def run(state):
    c = state["c"]
    if c["kind"] == "rope":
        ck, cv = state["cache"]
        if own:
            st = state["store"]
            st.set_len(0, c["n0"])
            st.append_rope(0, state["q"], state["k"], state["v"], state["rope"], positions=state["positions"], q_out=state["out"])
            return state["out"], ck, cv
        angle = state["positions"][..., state["axis"]].double() * state["frequencies"]
        ck.copy_(_turn(state["k"], angle, c["adjacent"]).transpose(1, 2).reshape(ck.shape))
        cv.copy_(state["v"].transpose(1, 2).reshape(cv.shape))
        return _turn(state["q"], angle, c["adjacent"]), ck, cv
    if c["kind"] == "pack":
        if own:
            st, last = state["store"], c["first"] + c["chunks"]
            st.pack_chunks(0, c["first"], last)
            return st.unpack_chunks(0, c["first"], last)
        return tuple(_from4(*_to4(state[x][:, state["rows"]])).to(torch.bfloat16) for x in ("k", "v"))
    B, T, Hq, Hkv = c["B"], c["T"], c["Hq"], c["Hkv"]
    if own:
        lse = torch.empty(B, T, Hq, dtype=torch.float32, device=DEV)
        return state["store"].decode_attn_q4(0, state["q"], dense=not c["gated"], causal=c["causal"], lse=lse), lse
    k, v = (torch.cat([_from4(*state[x + "4"]), state[x + "16"].float()], dim=1) for x in ("k", "v"))
    q = state["q"].float().view(B, T, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(B * Hkv, T * (Hq // Hkv), D)
    logits = (q @ k.transpose(1, 2)) * SCALE
    if c["gated"]:
        hidden = (state["scores"] < state["tau"]).repeat_interleave(c["C"], dim=1)
        logits[:, :, :state["split"]].masked_fill_(hidden.unsqueeze(1), -math.inf)
    if c["causal"]:
        last = c["n"] - T + torch.arange(T, device=DEV).repeat_interleave(Hq // Hkv)
        logits.masked_fill_(torch.arange(c["n"], device=DEV) > last.unsqueeze(1), -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    whole = lambda x: x.view(B, Hkv, T, Hq // Hkv, -1).transpose(1, 2).reshape(B, T, Hq, -1)
    return whole((p @ v) / total).to(torch.bfloat16), whole(top + torch.log(total)).squeeze(-1)


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------------------------

def _values_of(rows):
    """what 4 bits keep of [rows, 128], one group of 64 at a time, counted border by border"""
    kept = torch.empty(rows.shape, dtype=torch.float64, device=rows.device)
    for g in (slice(0, 64), slice(64, 128)):
        x = rows[:, g].double()
        low = x.min(dim=1, keepdim=True).values
        scale = (x.max(dim=1, keepdim=True).values - low) / 15
        mantissa, exponent = torch.frexp(scale)
        scale = torch.ldexp(torch.round(mantissa * 256), exponent - 8)
        code = torch.zeros_like(x)
        for k in range(15):
            code += (x - low > (k + 0.5) * scale) & (scale > 0)
        kept[:, g] = low + code * scale
    return kept


def exact(case, seed):
    c = case
    if c["kind"] == "rope":
        q, k, v, positions = _rope_inputs(c, seed)
        frequencies, axis, _ = _frequencies(c["axes"])
        turns = torch.stack([positions[..., a].double() * f for f, a in zip(frequencies, axis)], dim=-1)
        turns = torch.polar(torch.ones_like(turns), turns).unsqueeze(2)

        def turned(x):
            x = x.double()
            pairs = x.unflatten(-1, (64, 2)) if c["adjacent"] else x.unflatten(-1, (2, 64)).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turns)
            return (y if c["adjacent"] else y.transpose(-1, -2)).flatten(-2)
        by_sequence = lambda x: x.transpose(1, 2).flatten(0, 1)
        return turned(q), by_sequence(turned(k)), by_sequence(v.double())
    if c["kind"] == "pack":
        n = (c["first"] + c["chunks"]) * c["C"]
        k, v, _ = _cache_inputs(c, seed, c["B"] * c["H"], n, c["C"])
        return tuple(torch.stack([_values_of(s[c["first"] * c["C"]:]) for s in x]) for x in (k, v))
    k, v, q, scores, tau = _attn_inputs(c, seed)
    B, T, Hq, Hkv, nc = c["B"], c["T"], c["Hq"], c["Hkv"], _stale(c)
    G, split = Hq // Hkv, nc * c["C"]
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, T, Hq, dtype=torch.float64, device=DEV)
    position = torch.arange(c["n"], device=DEV)
    for s in range(B * Hkv):
        seen = torch.ones(c["n"], dtype=torch.bool, device=DEV)
        if c["gated"]:
            seen[:split] = (scores[s] >= tau).repeat_interleave(c["C"])
        keys, values = (torch.cat([_values_of(x[s, :split]), x[s, split:].double()])[seen] for x in (k, v))
        where = position[seen]
        heads = slice(s % Hkv * G, s % Hkv * G + G)
        for t in range(T):
            logits = q[s // Hkv, t, heads].double() @ keys.T / math.sqrt(D)
            if c["causal"]:
                logits[:, where > c["n"] - T + t] = -math.inf
            lse[s // Hkv, t, heads] = torch.logsumexp(logits, dim=-1)
            out[s // Hkv, t, heads] = torch.softmax(logits, dim=-1) @ values
    return out, lse
