"""Attention over a bounded view of the prefix cache: the calls that are measured.

Four operators of one path, a cache that stays small while the prefix grows:

* attention of draft slots with a sliding window over the committed prefix and
  a few first tokens that stay visible (`slot_attn` with `window` and `sinks`);
* attention of draft slots over a cache held in 4 bits (`slot_attn_q4`, with or
  without a window);
* the accepted tokens' keys and values appended to the 4-bit cache
  (`kv_append_q4`);
* a prefix of keys and values put into the 4-bit cache and taken out of it
  (`kv_quantize`, `kv_dequantize`).

The 4-bit cache holds blocks of 32 neighbouring elements of a head's row: 32
codes e2m1 (sign, and a magnitude of 0, 1/2, 1, 3/2, 2, 3, 4 or 6; the lower
element of a byte in its low bits) and one power of two 2^(byte - 127), the
smallest for which the block's largest magnitude rounds to at most 6; a byte of
255 marks a block that held a NaN or an infinity.

Sizes are those of `workloads/` (the 0.6B, 1.7B and 4B heads, prefixes, slots and
the training layout), of single tokens and single sequences beside them, and of
ranges around both.  Values are N(0, 1), as in `workloads/`; a prefix to be
quantised has channels of different sizes, as keys have.  With `own` the passes
are the framework's calls, otherwise elementary torch operations in float32.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ the cases


def _attn(name, kind, B, heads, P, S, L, D=128, dtype="bf16", ar=False, causal=False, ragged=False, W=0, sinks=0):
    return dict(name=name, kind=kind, dtype=dtype, B=B, Hq=heads[0], Hkv=heads[1], D=D, P=P, S=S, L=L, ar=ar,
                causal=causal, ragged=ragged, W=W, sinks=sinks)


def listed():
    return [
        # one interactive sequence that decodes token by token under a window:
        # the smallest call, where launches and idle units count
        _attn("window_token_single", "window", 1, (16, 8), 2048, 1, 1, W=512, sinks=4),
        # draft slots of the 4B serving batch under a window of a quarter of the prefix
        _attn("window_draft_4b", "window", 8, (32, 8), 16384, 8, 16, ragged=True, W=4096, sinks=4),
        # training layout of a model with sliding-window layers: 4096 tokens, no cache
        _attn("window_layout", "window", 8, (16, 8), 0, 128, 32, ar=True, causal=True, W=1024, sinks=4),
        # a reference-precision run of a small batch, odd lengths
        _attn("window_f32", "window", 2, (16, 8), 1000, 8, 8, dtype="f32", ragged=True, W=301, sinks=5),
        # one long-context sequence, one token: few rows over a long 4-bit cache
        _attn("q4_token_single", "q4", 1, (32, 8), 16384, 1, 1),
        # a serving batch that decodes token by token over long ragged caches:
        # the cache's bytes are all that counts
        _attn("q4_token_batch", "q4", 64, (16, 8), 8191, 1, 1, ragged=True),
        # draft slots of the 4B serving batch (the headline step's attention)
        _attn("q4_draft_4b", "q4", 8, (32, 8), 16384, 8, 16),
        # verification of a 1.7B serving batch, both savings together
        _attn("q4_window_verify_1.7b", "q4", 32, (16, 8), 4093, 16, 4, ar=True, ragged=True, W=1024, sinks=4),
        # the tokens that one sequence has accepted, in float32
        dict(name="append_single_f32", kind="append", dtype="f32", B=1, Hkv=8, D=64, C=333, P=300, S=4, L=8),
        # the tokens that a 0.6B serving batch has accepted
        dict(name="append_0.6b", kind="append", dtype="bf16", B=16, Hkv=8, D=128, C=2304, P=2048, S=8, L=8),
        # a short prompt of one sequence in float32, odd lengths
        dict(name="quantize_prompt_f32", kind="quantize", dtype="f32", B=1, Hkv=8, D=64, C=1025, N=777),
        # the prompts of the 4B serving batch
        dict(name="quantize_prompts_4b", kind="quantize", dtype="bf16", B=8, Hkv=8, D=128, C=16640, N=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_attn(rng):
    while True:
        kind = rng.choice(["window", "q4"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        heads = rng.choice([(16, 8), (32, 8), (16, 8), (12, 4), (8, 8), (7, 1)])
        layout = kind == "window" and rng.random() < 0.15
        P = 0 if layout else _log_int(rng, 17, 16384 if dtype == "bf16" else 2048)
        if layout:
            S, L = _log_int(rng, 8, 128), _log_int(rng, 4, 32)
        else:
            S, L = rng.choice([(1, 1), (1, 1), (_log_int(rng, 1, 16), _log_int(rng, 1, 24))])
        W = _log_int(rng, 16, 4096) if kind == "window" or rng.random() < 0.4 else 0
        c = _attn("", kind, _log_int(rng, 1, 64 if dtype == "bf16" else 4), heads, P, S, L,
                  D=rng.choice([128, 128, 64]), dtype=dtype, ar=rng.random() < 0.5,
                  causal=layout or rng.random() < 0.2, ragged=P > 0 and rng.random() < 0.6, W=W,
                  sinks=rng.choice([0, 1, 4, 4, 70]) if W else 0)
        w = work(c)
        if w["flops"] <= (2.5e11 if dtype == "bf16" else 1e9) and w["bytes"] <= 1e9 and _scores(c) <= 2.2e9:
            return c


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "append", "quantize"])
    if kind == "attn":
        c = _draw_attn(rng)
    else:
        dtype, D = rng.choice(["bf16", "bf16", "f32"]), rng.choice([128, 128, 64])
        Hkv = rng.choice([8, 8, 4, 3, 1])
        if kind == "append":
            S, L, P = _log_int(rng, 1, 24), _log_int(rng, 1, 24), _log_int(rng, 16, 4096)
            c = dict(name="", kind=kind, dtype=dtype, B=_log_int(rng, 1, 24), Hkv=Hkv, D=D,
                     C=P + rng.randint(0, S * L + 40), P=P, S=S, L=L)
        else:
            N = _log_int(rng, 1, 16384)
            c = dict(name="", kind=kind, dtype=dtype, B=_log_int(rng, 1, 8 if dtype == "bf16" else 4), Hkv=Hkv, D=D,
                     C=N + rng.randint(0, 300), N=N)
    del c["name"]
    return c


def _scores(c):
    """Scores of the whole prefix, masked ones included."""
    T = c["S"] * c["L"]
    return c["B"] * c["Hq"] * T * (c["P"] + T)


def _lens(c):
    """Prefix lengths of a case's rows: all P, or spread evenly from P/2 to P."""
    B, P = c["B"], c["P"]
    if not c["ragged"] or B == 1:
        return [P] * B
    return [P - (P - P // 2) * i // (B - 1) for i in range(B)]


# ------------------------------------------------------------------ the states


def _normal(g, shape, dtype, channels=None):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    rows = out.view(-1, shape[-1])
    step = max(1, (1 << 26) // shape[-1])
    for i in range(0, rows.shape[0], step):  # in pieces: the float32 draw of a large tensor is never whole
        x = torch.randn(rows[i:i + step].shape, generator=g, device="cuda")
        rows[i:i + step] = x if channels is None else x * channels
    return out


def _codes(x):
    """(codes, scale bytes) of finite float32 rows [..., D]."""
    blocks = x.unflatten(-1, (-1, BLOCK))
    bits = blocks.abs().amax(-1).view(torch.int32)
    # exponent of the largest magnitude, less 2 (6 = 1.5 * 2^2); one more from 1.75 on, which rounds to 8
    byte = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) >= 0x600000).int()).clamp(0, 252)
    unit = torch.exp2(127.0 - byte.float()).unsqueeze(-1)
    a = blocks.abs() * unit
    # to the nearest magnitude, halfway to the one whose code is even
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * (blocks < 0)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _values(codes, scales):
    """float32 values [..., D] of codes [..., D/2] and scale bytes [..., D/32]."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, BLOCK)) * torch.exp2(scales.float() - 127.0).unsqueeze(-1)).flatten(-2)


def _packed(g, shape):
    """(codes, scales) of N(0, 1) rows, in pieces."""
    D = shape[-1]
    codes = torch.empty(shape[:-1] + (D // 2,), dtype=torch.uint8, device="cuda")
    scales = torch.empty(shape[:-1] + (D // BLOCK,), dtype=torch.uint8, device="cuda")
    c, s = codes.view(-1, D // 2), scales.view(-1, D // BLOCK)
    step = (1 << 25) // D
    for i in range(0, c.shape[0], step):
        c[i:i + step], s[i:i + step] = _codes(torch.randn((min(step, c.shape[0] - i), D), generator=g, device="cuda"))
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, dt = case, DTYPES[case["dtype"]]
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    s = dict(case=c)  # "cache": codes and scales of the keys, then of the values
    if c["kind"] in ("window", "q4"):
        T = c["S"] * c["L"]
        s["q"] = _normal(g, (B, c["Hq"], T, D), dt)
        s["k_slot"], s["v_slot"] = _normal(g, (B, Hkv, T, D), dt), _normal(g, (B, Hkv, T, D), dt)
        lens = torch.tensor(_lens(c), device="cuda")[torch.randperm(B, generator=g, device="cuda")]
        s["lens"] = lens.to(torch.int32)
        if c["P"] and c["kind"] == "window":
            s["k_cache"], s["v_cache"] = _normal(g, (B, Hkv, c["P"], D), dt), _normal(g, (B, Hkv, c["P"], D), dt)
        elif c["P"]:
            s["cache"] = _packed(g, (B, Hkv, c["P"], D)) + _packed(g, (B, Hkv, c["P"], D))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, c["Hq"], T), device="cuda")
    elif c["kind"] == "append":
        S, L = c["S"], c["L"]
        s["cache"] = _packed(g, (B, Hkv, c["C"], D)) + _packed(g, (B, Hkv, c["C"], D))
        s["k_slot"], s["v_slot"] = _normal(g, (B, Hkv, S * L, D), dt), _normal(g, (B, Hkv, S * L, D), dt)
        s["lens0"] = torch.randint(c["P"] // 2, c["P"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        s["lens"] = s["lens0"].clone()
        # the verified slots in their order, then -1; a leading run of each is accepted
        n = torch.randint(1, S + 1, (B, 1), generator=g, device="cuda")
        order = torch.rand((B, S), generator=g, device="cuda").argsort(1)
        s["order"] = torch.where(torch.arange(S, device="cuda") < n, order, -1).to(torch.int32)
        run = torch.randint(0, L + 1, (B, S, 1), generator=g, device="cuda")
        s["accepted"] = (torch.arange(L, device="cuda") < run).to(torch.uint8)
    else:
        size = torch.exp(0.5 * torch.randn(D, generator=g, device="cuda"))
        s["k"], s["v"] = _normal(g, (B, Hkv, c["N"], D), dt, size), _normal(g, (B, Hkv, c["N"], D), dt)
        s["cache"] = tuple(torch.zeros((B, Hkv, c["C"], n), dtype=torch.uint8, device="cuda")
                           for n in (D // 2, D // BLOCK, D // 2, D // BLOCK))
    return s


# ------------------------------------------------------------------ the passes


def _visible(lens, P, S, L, ar, causal, W, sinks):
    """[B, T, P + T]: which keys, the prefix's and then the draft tokens', each draft token sees."""
    dev = lens.device
    t, j = torch.arange(S * L, device=dev), torch.arange(P, device=dev)
    n = lens.long().view(-1, 1, 1)
    same, earlier = t[:, None] // L == t // L, t[:, None] // L > t // L
    draft = same & (t <= t[:, None]) if ar else same
    if causal:
        draft = draft | earlier
    seen = torch.cat(((j < n).expand(-1, S * L, -1), draft.expand(n.shape[0], -1, -1)), 2)
    if W:
        at = torch.cat((j.expand(n.shape[0], 1, -1), n + t), 2)  # places in the committed order
        seen = seen & ((at < sinks) | (at > n + t[:, None] - W))
    return seen


def _attention(q, k, v, seen, G):
    """Softmax attention in float32; `seen` is the same for the G query heads of a key head."""
    B, Hq, T, D = q.shape
    x = q.float().view(B, Hq // G, G * T, D) @ k.transpose(-1, -2)
    x = (x * (1.0 / math.sqrt(D))).view(B, Hq // G, G, T, -1)
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ v).view(B, Hq // G, G, T, D) / total
    return out.reshape(B, Hq, T, D).to(q.dtype), (m + torch.log(total)).reshape(B, Hq, T)


def _plain_attn(s):
    c = s["case"]
    k, v = s["k_slot"].float(), s["v_slot"].float()
    if c["P"] and c["kind"] == "window":
        k, v = torch.cat((s["k_cache"].float(), k), 2), torch.cat((s["v_cache"].float(), v), 2)
    elif c["P"]:
        a = s["cache"]
        k, v = torch.cat((_values(a[0], a[1]), k), 2), torch.cat((_values(a[2], a[3]), v), 2)
    seen = _visible(s["lens"], c["P"], c["S"], c["L"], c["ar"], c["causal"], c["W"], c["sinks"])
    return _attention(s["q"], k, v, seen, c["Hq"] // c["Hkv"])


def _plain_append(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    B, Hkv, D, S, L, C = c["B"], c["Hkv"], c["D"], c["S"], c["L"], c["C"]
    order, n0 = s["order"].long(), s["lens0"].long()
    at = torch.full((B, S + 1), S, device="cuda").scatter(1, torch.where(order < 0, S, order),
                                                          torch.arange(S, device="cuda").expand(B, -1))[:, :S]
    taken = (s["accepted"] != 0) & (at < S)[:, :, None]
    rank = torch.where(taken, at[:, :, None] * L + torch.arange(L, device="cuda"), S * L).flatten(1)
    token = rank.argsort(1)  # the accepted tokens in append order, then the others
    n = taken.flatten(1).sum(1)
    n = torch.where(n0 + n > C, 0, n)  # a row that does not fit stays as it is
    place = torch.arange(C, device="cuda") - n0[:, None]
    new = (place >= 0) & (place < n[:, None])
    token = token.gather(1, place.clamp(0, S * L - 1))[:, None, :, None].expand(-1, Hkv, -1, D)
    k = _values(*_codes(s["k_slot"].float())).gather(2, token)
    v = _values(*_codes(s["v_slot"].float())).gather(2, token)
    a, new = s["cache"], new[:, None, :, None]
    return (torch.where(new, k, _values(a[0], a[1])).to(dt), torch.where(new, v, _values(a[2], a[3])).to(dt),
            (n0 + n).to(torch.int32))


def run(s):
    c = s["case"]
    if not own:
        if c["kind"] in ("window", "q4"):
            return _plain_attn(s)
        if c["kind"] == "append":
            return _plain_append(s)
        return tuple(_values(*_codes(x.float())).to(x.dtype) for x in (s["k"], s["v"]))

    import paper_2609_19868_amd as Z

    if c["kind"] in ("window", "q4"):
        how = dict(pass_=Z.PASS_AR_INFILL if c["ar"] else Z.PASS_DIFFUSION,
                   cross_slot=Z.CROSS_SLOT_CAUSAL if c["causal"] else Z.CROSS_SLOT_NONE, prefix_lens=s["lens"],
                   out=s["out"], lse=s["lse"], window=c["W"] or None, sinks=c["sinks"])
        if c["kind"] == "window":
            return Z.slot_attn(s["q"], s.get("k_cache"), s.get("v_cache"), s["k_slot"], s["v_slot"], c["S"], c["L"], **how)
        return Z.slot_attn_q4(s["q"], Z.Q4Cache(*s["cache"]), s["k_slot"], s["v_slot"], c["S"], c["L"], **how)
    cache = Z.Q4Cache(*s["cache"])
    if c["kind"] == "append":
        s["lens"].copy_(s["lens0"])  # so that a pass can be repeated
        Z.kv_append_q4(cache, s["lens"], s["k_slot"], s["v_slot"], s["accepted"], s["order"])
        return Z.kv_dequantize(cache, dtype=DTYPES[c["dtype"]]) + (s["lens"],)
    Z.kv_quantize(s["k"], s["v"], cache)
    return Z.kv_dequantize(cache, n_rows=c["N"], dtype=s["k"].dtype)


# ------------------------------------------------------------------ their work


def _seen_per_row(c, n):
    """Visible keys of each draft token and prefix rows that any of them sees, for a prefix of n rows."""
    S, L, W, sinks = c["S"], c["L"], c["W"] or 1 << 40, c["sinks"]
    T = S * L
    t = np.arange(T)
    low = np.maximum(n + t - W + 1, 0)  # first place inside the window
    prefix = n - np.minimum(low, n) + np.minimum(np.minimum(low, n), sinks)
    first = np.zeros(T, np.int64) if c["causal"] else t // L * L
    end = t + 1 if c["ar"] else (t // L + 1) * L
    low = np.clip(low - n, first, end)
    draft = end - low + np.clip(np.minimum(low, max(0, sinks - n)) - first, 0, None)
    union = n - min(max(n - W + 1, 0), n)
    return int((prefix + draft).sum()), union + min(n - union, sinks)


def work(case):
    c, size = case, 2 if case["dtype"] == "bf16" else 4
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    if c["kind"] in ("window", "q4"):
        T = c["S"] * c["L"]
        rows = [_seen_per_row(c, n) for n in _lens(c)]
        row = D * size if c["kind"] == "window" else D // 2 + D // BLOCK
        # the visible prefix rows once, the draft tokens' own K/V, Q and O, the log-sum-exps
        moved = 2 * Hkv * row * sum(r[1] for r in rows) + 2 * B * (Hkv + c["Hq"]) * T * D * size + 4 * B * c["Hq"] * T
        return {"bytes": moved, "flops": 4 * D * c["Hq"] * sum(r[0] for r in rows)}
    packed = D // 2 + D // BLOCK
    if c["kind"] == "append":
        S, L, C = c["S"], c["L"], c["C"]
        tokens = (S + 1) / 2 * L / 2  # accepted on average
        # the accepted rows in, the whole cache out as the values it stands for
        return {"bytes": 2 * B * Hkv * (tokens * D * size + C * packed + C * D * size) + B * S * (L + 4), "flops": 0}
    return {"bytes": 2 * B * Hkv * c["N"] * 2 * D * size, "flops": 0}


# ------------------------------------------------------------------ in 64 bits


def _exact_round(x):
    """The nearest value that a block of x (float64, [..., D]) has in 4 bits."""
    y = x.reshape(x.shape[:-1] + (-1, BLOCK))
    top = y.abs().max(-1, keepdim=True)[0]
    _, e = torch.frexp(torch.where(top > 0, top, torch.full_like(top, 2.0 ** -126)))  # top in [2^(e-1), 2^e)
    e = e.double() - 3
    e = torch.where(top >= 7 * 2.0 ** e, e + 1, e).clamp(-127, 125)
    scaled = y / 2.0 ** e
    # spacing of the magnitudes around a value: 1/2 below 2, 1 below 4, then 2 (torch rounds halves to even)
    a = scaled.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    near = (torch.round(a / step) * step).clamp(max=6.0)
    return (torch.sign(scaled) * near * 2.0 ** e).reshape(x.shape)


def _exact_unpack(codes, scales):
    both = torch.stack((codes % 16, codes // 16), -1).reshape(codes.shape[:-1] + (-1,)).long()
    e, m = both % 8 // 2, (both % 2).double()
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1).double())
    mag = torch.where(both >= 8, -mag, mag)
    return mag * torch.repeat_interleave(2.0 ** (scales.double() - 127), BLOCK, -1)


def _exact_row(c, q, k, v, ks, vs, n, out, lse):
    """One batch row: heads one after another, each over its visible keys in the order of their places."""
    S, L, W, sinks, G = c["S"], c["L"], c["W"], c["sinks"], c["Hq"] // c["Hkv"]
    T = S * L
    place_k = torch.arange(n + T, device="cuda")
    place_q = place_k[n:, None]
    slot_k, slot_q = (place_k - n).div(L, rounding_mode="floor"), (place_q - n) // L
    ok = (place_k < n) | (slot_k == slot_q) & ((place_k <= place_q) | (not c["ar"]))
    if c["causal"]:
        ok |= (place_k >= n) & (slot_k < slot_q)
    if W:
        ok &= (place_q - place_k < W) | (place_k < sinks)
    for h in range(c["Hkv"]):
        kk, vv = torch.cat((k[h, :n], ks[h])), torch.cat((v[h, :n], vs[h]))
        for i in range(h * G, h * G + G):
            z = torch.mm(q[i], kk.t().contiguous()) / math.sqrt(c["D"])
            z[~ok] = -math.inf
            lse[i] = torch.logsumexp(z, 1)
            out[i] = torch.mm(torch.exp(z - lse[i][:, None]), vv)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    if c["kind"] in ("window", "q4"):
        T = c["S"] * c["L"]
        out = torch.empty((B, c["Hq"], T, D), dtype=torch.float64, device="cuda")
        lse = torch.empty((B, c["Hq"], T), dtype=torch.float64, device="cuda")
        for b in range(B):
            if not c["P"]:
                k = v = torch.empty((Hkv, 0, D), dtype=torch.float64, device="cuda")
            elif c["kind"] == "window":
                k, v = s["k_cache"][b].double(), s["v_cache"][b].double()
            else:
                k, v = (_exact_unpack(s["cache"][i][b], s["cache"][i + 1][b]) for i in (0, 2))
            _exact_row(c, s["q"][b].double(), k, v, s["k_slot"][b].double(), s["v_slot"][b].double(),
                       int(s["lens"][b]), out[b], lse[b])
        return out, lse
    if c["kind"] == "quantize":
        return tuple(torch.cat([_exact_round(x[b:b + 1].double()) for b in range(B)]) for x in (s["k"], s["v"]))
    k, v = (_exact_unpack(s["cache"][i], s["cache"][i + 1]) for i in (0, 2))
    lens = s["lens0"].tolist()
    for b in range(B):
        tokens = []
        for slot in s["order"][b].tolist():
            if slot < 0:
                break
            tokens += [slot * c["L"] + r for r, a in enumerate(s["accepted"][b, slot].tolist()) if a]
        if tokens and lens[b] + len(tokens) <= c["C"]:
            k[b, :, lens[b]:lens[b] + len(tokens)] = _exact_round(s["k_slot"][b].double()[:, tokens])
            v[b, :, lens[b]:lens[b] + len(tokens)] = _exact_round(s["v_slot"][b].double()[:, tokens])
            lens[b] += len(tokens)
    return k, v, torch.tensor(lens, dtype=torch.int32, device="cuda")
