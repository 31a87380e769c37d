"""The operators between a decoder block's q/k/v projections and its output projection, as cases a
timing harness can run: normalising and rotating queries and keys, writing keys and values into a
cache of 8-bit floats, reading them back, and attention over that cache.

A case is a dict of plain values.  `prepare` makes what a user's program holds before the call, `run`
is one pass (the plain form in elementary torch operations, or with `own` the calls of
`paper_2604_03957_amd.binding`), `work` the bytes and operations one pass cannot do without, `exact`
the same outputs from the operators' definitions in 64 bits.

The cache: blocks of `block` tokens; codes are E4M3 and a block has one scale 2^e per head, for its
keys and for its values.  e is the smallest exponent with max |x| <= 448 * 2^e over the finite values
(at least -40, at most 40); a code is x * 2^-e rounded to the nearest E4M3 value.  A later token that
needs a larger e raises it, and the codes that are there are divided by the ratio and rounded again.
Keys lie as [blocks, kv_heads, block, dim], values as [blocks, kv_heads, dim, block].

Paths (`case["path"]`):
  rope       bwta_head_norm_rope on the q/k part of projected tokens
  write      bwta_cache_write of new tokens; where "back" is true, bwta_cache_read of the same tokens
  read       bwta_cache_read of whole sequences
  attention  bwta_cache_attention of new tokens over all that is cached
  step       one decode step: the three calls in a row, one token for each sequence
"""
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
FP8 = torch.float8_e4m3fn
E_MIN, E_MAX = -40, 40


def listed():
    return [
        # one generated token of a 7B decoder: 32 heads of 128
        {"name": "rope_token", "path": "rope", "M": 1, "heads": 32, "kv_heads": 32, "dim": 128, "rot": 128, "interleaved": False, "norm": True, "far": 4096, "dtype": "fp16"},
        # a long prompt of grouped heads whose q/k/v come from one projection, far into a document
        {"name": "rope_prompt", "path": "rope", "M": 8192, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128, "interleaved": False, "norm": True, "far": 1000000, "dtype": "bf16"},
        # a decode step's keys and values: 64 sequences, one token each
        {"name": "write_tokens", "path": "write", "batch": 64, "new": 1, "cached": 4096, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "fp16", "back": False},
        # prompts of several lengths into the cache, and back out of it (a check, or a move to another place)
        {"name": "write_prompts", "path": "write", "batch": 5, "new": 4001, "cached": 500, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "fp16", "back": True},
        # whole contexts back to 16 bits
        {"name": "read_contexts", "path": "read", "batch": 8, "len": 8000, "kv_heads": 8, "dim": 128, "block": 128, "dtype": "bf16"},
        # one token of one 7B sequence, 2048 tokens in
        {"name": "attention_token", "path": "attention", "batch": 1, "new": 1, "cached": 2047, "heads": 32, "kv_heads": 32, "dim": 128, "block": 64, "dtype": "fp16", "causal": True, "window": 0},
        # a serving batch of decode tokens, contexts of many lengths
        {"name": "attention_batch", "path": "attention", "batch": 64, "new": 1, "cached": 8191, "heads": 32, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "fp16", "causal": True, "window": 0},
        # one token of one very long sequence
        {"name": "attention_long", "path": "attention", "batch": 1, "new": 1, "cached": 131071, "heads": 32, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "bf16", "causal": True, "window": 0},
        # a 2048-token prompt of a 7B decoder
        {"name": "attention_prompt", "path": "attention", "batch": 1, "new": 2048, "cached": 0, "heads": 32, "kv_heads": 32, "dim": 128, "block": 64, "dtype": "fp16", "causal": True, "window": 0},
        # chunks of long prompts behind what is cached of them
        {"name": "attention_chunks", "path": "attention", "batch": 4, "new": 1024, "cached": 15000, "heads": 32, "kv_heads": 8, "dim": 128, "block": 128, "dtype": "bf16", "causal": True, "window": 0},
        # a decoder's tokens over an encoder's states: every query sees every key
        {"name": "attention_encoder", "path": "attention", "batch": 32, "new": 128, "cached": 200, "heads": 12, "kv_heads": 12, "dim": 64, "block": 64, "dtype": "fp16", "causal": False, "window": 0},
        # a decode step from the projections to the attention's output
        {"name": "step_batch", "path": "step", "batch": 32, "new": 1, "cached": 3000, "heads": 32, "kv_heads": 8, "dim": 128, "block": 64, "dtype": "fp16", "causal": True, "window": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    path = rng.choice(["rope", "write", "read", "attention", "attention", "attention", "attention", "step"])
    while True:
        kv = rng.choice([1, 2, 4, 8, 12, 32])
        c = {"path": path, "kv_heads": kv, "dim": rng.choice([64, 128, 128, 256]), "dtype": rng.choice(["fp16", "bf16"])}
        if path == "rope":
            c.update(M=_log_int(rng, 1, 8192), heads=kv * rng.choice([1, 2, 4, 5, 8]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.8, far=_log_int(rng, 1, 1000000))
            c["rot"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2])
            ok = c["M"] * (c["heads"] + kv) * c["dim"] <= 8192 * 40 * 128
        elif path == "write":
            c.update(batch=_log_int(rng, 1, 64), new=_log_int(rng, 1, 4001), cached=_log_int(rng, 1, 4096), block=rng.choice([64, 128, 256]), back=rng.random() < 0.5)
            ok = c["batch"] * c["new"] * kv * c["dim"] <= 5 * 4001 * 8 * 128 and c["batch"] * (c["new"] + c["cached"]) * kv * c["dim"] <= 64 * 4096 * 8 * 128
        elif path == "read":
            c.update(batch=_log_int(rng, 1, 64), len=_log_int(rng, 1, 16384), block=rng.choice([64, 128, 256]))
            ok = c["batch"] * c["len"] * kv * c["dim"] <= 8 * 8000 * 8 * 128
        else:
            c.update(batch=_log_int(rng, 1, 64), new=1, cached=_log_int(rng, 1, 131071), heads=kv * rng.choice([1, 2, 4, 5, 8]), block=rng.choice([64, 128, 256]),
                     causal=True, window=0)
            if path == "attention":
                if rng.random() < 0.5:
                    c["new"] = _log_int(rng, 2, 4096)
                c["causal"] = rng.random() < 0.8
                if c["causal"] and rng.random() < 0.25:
                    c["window"] = _log_int(rng, 16, 4096)
            keys = c["new"] + c["cached"]
            ok = (c["heads"] <= 64 and c["batch"] * keys * kv * c["dim"] <= 64 * 8192 * 8 * 128
                  and c["batch"] * c["new"] * keys * c["heads"] <= 4 * 1024 * 16000 * 32)
        if ok:
            return c


# ---- inputs --------------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _lengths(case):
    """(tokens of the call, tokens cached with them) of each sequence: of several sizes, the first the largest.  They follow
    from the case alone."""
    rng = random.Random("%d %d" % (case["batch"], case["kv_heads"]))
    new, lens = [], []
    for b in range(case["batch"]):
        if case["path"] == "read":
            n = case["len"] if b == 0 else rng.randint((case["len"] + 3) // 4, case["len"])
            c = 0
        else:
            n = case["new"] if b == 0 else rng.randint((case["new"] + 1) // 2, case["new"])
            c = case["cached"] if b == 0 else rng.randint(case["cached"] // 4, case["cached"])
        new.append(n)
        lens.append(n + c)
    return new, lens


def _rows(g, *shape, dtype, spread=True):
    """Projected heads: N(0, 1), some channels of keys several times as large, as trained models have them."""
    x = torch.randn(shape, device=DEV, generator=g)
    if spread:
        x = x * (1.0 + 4.0 * (torch.rand(shape[-2:], device=DEV, generator=g) < 0.05))
    return x.to(dtype)


def _cache(case, g, lens):
    """The cache a program holds: blocks in any order, with all but the last `new` tokens of each sequence written.  The
    contents are codes of N(0, 1) values with a few larger channels, each block with a scale of its own."""
    H, D, blk = case["kv_heads"], case["dim"], case["block"]
    wide = -(-max(lens) // blk)
    spare = 3
    total = sum(-(-n // blk) for n in lens) + spare
    order = torch.randperm(total, device=DEV, generator=g).to(torch.int32)
    table = torch.zeros((len(lens), wide), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(lens):
        need = -(-n // blk)
        table[b, :need] = order[at:at + need]
        at += need
    state = {"table": table}
    for name, shape in (("k", (total, H, blk, D)), ("v", (total, H, D, blk))):
        state[name] = torch.empty(shape, dtype=torch.uint8, device=DEV)
        state[name + "_scale"] = torch.empty((total, H), dtype=torch.float32, device=DEV)
        step = max(1, (1 << 27) // (H * D * blk))
        for at in range(0, total, step):
            part = slice(at, min(total, at + step))
            n = part.stop - part.start
            x = torch.randn((n,) + shape[1:], device=DEV, generator=g)
            x = x * torch.exp2(torch.randint(-2, 3, (n, H, 1, 1), device=DEV, generator=g).float())
            e = _exponent(x.abs().amax(dim=(2, 3)))
            state[name + "_scale"][part] = torch.exp2(e)
            state[name][part] = (x * torch.exp2(-e)[:, :, None, None]).clamp(-448, 448).to(FP8).view(torch.uint8)
    return state


def _sequences(new, lens):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"lens": i32(lens), "cu": i32(cu), "M": cu[-1], "max_new": max(new), "max_len": max(lens), "new": new, "total": lens}


def _rope_state(case, g, M):
    dt, D, Hq, Hk = DTYPES[case["dtype"]], case["dim"], case["heads"], case["kv_heads"]
    qkv = _rows(g, M, Hq + 2 * Hk, D, dtype=dt)
    weight = lambda: (1.0 + 0.2 * torch.randn(D, device=DEV, generator=g)).to(dt)  # noqa: E731
    rot = case.get("rot", D)
    return {"qkv": qkv, "q": qkv[:, :Hq], "k_new": qkv[:, Hq:Hq + Hk], "v_new": qkv[:, Hq + Hk:], "wq": weight(), "wk": weight(),
            "inv_freq": (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)).float(),
            "q_out": torch.zeros((M, Hq, D), dtype=dt, device=DEV), "k_out": torch.zeros((M, Hk, D), dtype=dt, device=DEV)}


def prepare(case, seed):
    g = _gen(seed)
    dt, path = DTYPES[case["dtype"]], case["path"]
    s = {"case": case}
    if path == "rope":
        s.update(_rope_state(case, g, case["M"]))
        s["positions"] = (torch.arange(case["M"], device=DEV) + torch.randint(0, case["far"], (1,), device=DEV, generator=g)).to(torch.int32)
        return s
    new, lens = _lengths(case)
    s.update(_sequences(new, lens))
    s.update(_cache(case, g, lens))
    M, H, D = s["M"], case["kv_heads"], case["dim"]
    if path in ("write", "read"):
        s["k_new"], s["v_new"] = _rows(g, M, H, D, dtype=dt), _rows(g, M, H, D, dtype=dt, spread=False)
        s["k_out"], s["v_out"] = (torch.zeros((M, H, D), dtype=dt, device=DEV) for _ in range(2))
        return s
    Hq = case["heads"]
    if path == "step":
        s.update(_rope_state(case, g, M))
        s["positions"] = s["lens"] - 1
        s["v_new"] = s["v_new"].contiguous()
    else:
        s["q"] = _rows(g, M, Hq, D, dtype=dt)
    s["out"] = torch.zeros((M, Hq, D), dtype=dt, device=DEV)
    s["lse"] = torch.zeros((M, Hq), dtype=torch.float32, device=DEV)
    return s


# ---- the plain forms ------------------------------------------------------------------------------


def _exponent(amax):
    """The smallest whole e with amax <= 448 * 2^e, within the cache's range."""
    m, e = torch.frexp(amax.double())
    return torch.where(amax > 0, e - 9 + (m > 0.875), E_MIN).clamp(E_MIN, E_MAX).float()


def _plain_rope(s, x, w, positions):
    """x [M, heads, dim] -> normalised by head, times w, rotated by position."""
    c = s["case"]
    y = x.float()
    if c.get("norm", True):
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
    a = positions.double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    rot = c.get("rot", c["dim"])
    head, rest = y[..., :rot], y[..., rot:]
    if c.get("interleaved", False):
        u, v = head[..., 0::2], head[..., 1::2]
        head = torch.stack((u * cos - v * sin, u * sin + v * cos), dim=-1).flatten(-2)
    else:
        u, v = head[..., :rot // 2], head[..., rot // 2:]
        head = torch.cat((u * cos - v * sin, u * sin + v * cos), dim=-1)
    return torch.cat((head, rest), dim=-1).to(x.dtype)


def _token_places(s):
    """(sequence, position) of each token of the call."""
    t = torch.arange(s["M"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["cu"][1:].contiguous(), t, right=True)
    return seq, (s["lens"][seq] - s["cu"][seq + 1] + t).long()


def _plain_write_one(s, codes, scales, x, tokens_last):
    """codes [blocks, H, ...] seen with tokens in dimension 2 (`tokens_last` false) or 3; x [M, H, D]."""
    c = s["case"]
    blk = c["block"]
    seq, pos = _token_places(s)
    page, slot = s["table"][seq, pos // blk].long(), pos % blk
    x = x.float()
    finite = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dim=-1)
    need = torch.zeros_like(scales).scatter_reduce_(0, page[:, None].expand_as(finite), finite, "amax")
    starts = torch.zeros(scales.shape[0], device=DEV).index_fill_(0, page, 1.0)
    begun = torch.zeros(scales.shape[0], device=DEV).scatter_reduce_(0, page, (slot == 0).float(), "amax")
    asked = torch.exp2(_exponent(need))
    fresh = torch.where(begun[:, None] > 0, asked, torch.maximum(asked, scales))
    scale = torch.where(starts[:, None] > 0, fresh, scales)
    # the codes that are there, of the blocks that the call touches
    span = (s["max_new"] + blk - 2) // blk + 1
    first = ((s["lens"] - (s["cu"][1:] - s["cu"][:-1])) // blk).long()
    touched = first[:, None] + torch.arange(span, device=DEV)
    last = ((s["lens"] - 1) // blk).long()
    touched = s["table"].gather(1, torch.minimum(touched, last[:, None])).long().flatten()
    old = codes[touched].view(FP8).float()
    ratio = torch.where(begun[touched, None] > 0, 1.0, scales[touched] / scale[touched])[:, :, None, None]
    codes[touched] = (old * ratio).to(FP8).view(torch.uint8)
    y = torch.where(torch.isnan(x), 0.0, x / scale[page][:, :, None]).clamp(-448, 448).to(FP8).view(torch.uint8)
    if tokens_last:
        codes[page, :, :, slot] = y
    else:
        codes[page, :, slot] = y
    scales.copy_(scale)


def _plain_write(s, k, v):
    _plain_write_one(s, s["k"], s["k_scale"], k, False)
    _plain_write_one(s, s["v"], s["v_scale"], v, True)


def _plain_read(s):
    dt = DTYPES[s["case"]["dtype"]]
    blk, most = s["case"]["block"], torch.finfo(dt).max
    seq, pos = _token_places(s)
    page, slot = s["table"][seq, pos // blk].long(), pos % blk
    k = s["k"][page, :, slot].view(FP8).float() * s["k_scale"][page][:, :, None]
    v = s["v"][page, :, :, slot].view(FP8).float() * s["v_scale"][page][:, :, None]
    return k.clamp(-most, most).to(dt), v.clamp(-most, most).to(dt)


def _plain_attention(s, q):
    c = s["case"]
    B, H, D, G, T = c["batch"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"], s["max_new"]
    table = s["table"].long()
    k = (s["k"][table].view(FP8).float() * s["k_scale"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    v = (s["v"][table].view(FP8).float() * s["v_scale"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, H, -1, D)
    seq, pos = _token_places(s)
    t = torch.arange(s["M"], device=DEV) - s["cu"][seq]
    qs = torch.zeros((B, T, H, G, D), device=DEV)
    qs[seq, t] = q.float().view(-1, H, G, D)
    scores = torch.matmul(qs.permute(0, 2, 3, 1, 4).reshape(B, H, G * T, D), k.transpose(2, 3).contiguous()).view(B, H, G, T, -1)
    scores *= D ** -0.5
    key = torch.arange(k.shape[2], device=DEV)
    at = torch.zeros((B, T), dtype=torch.int64, device=DEV)
    at[seq, t] = pos
    hide = key >= s["lens"][:, None, None]
    if c["causal"]:
        hide = hide | (key > at[:, :, None])
    if c["window"]:
        hide = hide | (key <= at[:, :, None] - c["window"])
    scores.masked_fill_(hide[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, H, G * T, -1), v).view(B, H, G, T, D) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, T, H * G, D)[seq, t]
    return out.to(q.dtype), lse.permute(0, 3, 1, 2).reshape(B, T, H * G)[seq, t]


# ---- one pass --------------------------------------------------------------------------------------


def _held(s):
    """The cache's contents: the codes as the values they stand for in units of their scale, and the scales."""
    return {"k": s["k"].view(FP8), "v": s["v"].view(FP8), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _own(s):
    from paper_2604_03957_amd import binding as B
    c = s["case"]
    path, D = c["path"], c["dim"]
    if path in ("rope", "step"):
        B.bwta_head_norm_rope(s["q"], s["k_new"], s["wq"], s["wk"], s["positions"], s["inv_freq"], s["q_out"], s["k_out"], M=s["q"].shape[0], heads=c["heads"],
                              kv_heads=c["kv_heads"], dim=D, rot_dim=c.get("rot", D), eps=1e-6, norm=c.get("norm", True), interleaved=c.get("interleaved", False),
                              ldq=s["q"].stride(0), ldk=s["k_new"].stride(0))
        if path == "rope":
            return {"q": s["q_out"], "k": s["k_out"]}
    if "cache" not in s:
        s["cache"] = B.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    seqs = dict(M=s["M"], batch=c["batch"], max_new=s["max_new"], max_len=s["max_len"])
    if path in ("write", "step"):
        k = s["k_out"] if path == "step" else s["k_new"]
        B.bwta_cache_write(s["cache"], k, s["v_new"], s["table"], s["lens"], s["cu"], **seqs)
        if path == "write" and not c["back"]:
            return _held(s)
    if path in ("write", "read"):
        B.bwta_cache_read(s["cache"], s["k_out"], s["v_out"], s["table"], s["lens"], s["cu"], **seqs)
        got = {"k_back": s["k_out"], "v_back": s["v_out"]}
        return got if path == "read" else {**_held(s), **got}
    if "workspace" not in s:
        n = B.cache_attention_workspace_bytes(heads=c["heads"], kv_heads=c["kv_heads"], dim=D, **seqs)
        s["workspace"] = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    q = s["q_out"] if path == "step" else s["q"]
    B.bwta_cache_attention(s["cache"], q, s["out"], s["lse"], s["table"], s["lens"], s["cu"], s["workspace"], heads=c["heads"], alpha=D ** -0.5, causal=c["causal"],
                           window=c["window"], **seqs)
    got = {"out": s["out"], "lse": s["lse"]}
    return got if path == "attention" else {**_held(s), **got}


def run(s):
    if own:
        return _own(s)
    path = s["case"]["path"]
    if path in ("rope", "step"):
        q, k = _plain_rope(s, s["q"], s["wq"], s["positions"]), _plain_rope(s, s["k_new"], s["wk"], s["positions"])
        if path == "rope":
            return {"q": q, "k": k}
    if path in ("write", "step"):
        _plain_write(s, k if path == "step" else s["k_new"], s["v_new"])
        if path == "write" and not s["case"]["back"]:
            return _held(s)
    if path in ("write", "read"):
        k, v = _plain_read(s)
        return {"k_back": k, "v_back": v} if path == "read" else {**_held(s), "k_back": k, "v_back": v}
    out, lse = _plain_attention(s, q if path == "step" else s["q"])
    return {"out": out, "lse": lse} if path == "attention" else {**_held(s), "out": out, "lse": lse}


# ---- work ------------------------------------------------------------------------------------------


def _pairs(case):
    """(query, key) pairs one head sees, and the keys any query of each sequence sees, over all sequences."""
    new, lens = _lengths(case)
    pairs = keys = 0
    for n, m in zip(new, lens):
        if not case["causal"]:
            pairs, keys = pairs + n * m, keys + m
            continue
        w = case["window"] or m
        ramp = max(0, min(n, w - (m - n)))  # queries that see everything before them
        first = m - n + 1
        pairs += ramp * first + ramp * (ramp - 1) // 2 + (n - ramp) * w
        keys += min(m, w + n - 1)
    return pairs, keys


def work(case):
    path, D, H = case["path"], case["dim"], case["kv_heads"]
    if path == "rope":
        n = case["M"] * (case["heads"] + H) * D
        return {"bytes": 4.0 * n + 4.0 * case["M"] + 4.0 * D + 2.0 * case["rot"], "flops": 10.0 * n}
    new, lens = _lengths(case)
    M = sum(new)
    n = 2 * M * H * D  # keys and values
    table = 4.0 * sum(-(-m // case["block"]) for m in lens)
    if path == "write":
        return {"bytes": 3.0 * n + (3.0 * n if case["back"] else 0.0), "flops": 2.0 * n}
    if path == "read":
        return {"bytes": 3.0 * n + table, "flops": 1.0 * n}
    pairs, keys = _pairs(case)
    q = M * case["heads"] * D
    b = 2.0 * keys * H * D + 8.0 * keys / case["block"] * H + 4.0 * q + 4.0 * M * case["heads"] + table
    f = 4.0 * D * case["heads"] * pairs
    if path == "step":
        b, f = b + 4.0 * (q + n / 2) + 3.0 * n, f + 10.0 * (q + n / 2)
    return {"bytes": b, "flops": f}


# ---- the definitions in 64 bits --------------------------------------------------------------------


def _e4m3(x):
    """The nearest E4M3 value (ties to even) of x within +-448."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_rope(s, x, w):
    c = s["case"]
    x = x.double()
    if c.get("norm", True):
        x = x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
    rot, y = c.get("rot", c["dim"]), x.clone()
    i = torch.arange(rot // 2, device=DEV)
    a, b = (2 * i, 2 * i + 1) if c.get("interleaved", False) else (i, i + rot // 2)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(x.shape[0], rot // 2).contiguous(), s["positions"].double()[:, None] * s["inv_freq"].double())
    z = torch.complex(x[..., a], x[..., b]) * turn[:, None]
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_write(s, name, x):
    """One sequence after the other; the cache's values and scales in 64 bits."""
    codes, scales = s[name].view(FP8).double(), s[name + "_scale"].double()
    if name == "v":
        codes = codes.transpose(2, 3)
    codes, blk = codes.contiguous(), s["case"]["block"]
    at = 0
    for b, (n, m) in enumerate(zip(s["new"], s["total"])):
        p = m - n
        while p < m:
            page, lo = int(s["table"][b, p // blk]), p % blk
            take = min(m - p, blk - lo)
            new = x[at:at + take].double().transpose(0, 1)  # [H, take, D]
            top = new.abs().amax(dim=(1, 2))
            mant, e = torch.frexp(top / 448.0)
            e = torch.where(mant == 0.5, e - 1, e)
            scale = torch.exp2(torch.where(top > 0, e, E_MIN).clamp(E_MIN, E_MAX).double())
            if lo:
                scale = torch.maximum(scale, scales[page])
                codes[page] = _e4m3(codes[page] * (scales[page] / scale)[:, None, None])
            codes[page][:, lo:lo + take] = _e4m3(new / scale[:, None, None])
            scales[page] = scale
            at, p = at + take, p + take
    return (codes.transpose(2, 3) if name == "v" else codes), scales


def _exact_heads(s, name, b, codes=None, scales=None):
    """[H, tokens, D] of sequence b in 64 bits."""
    n = s["total"][b]
    pages = s["table"][b, :-(-n // s["case"]["block"])].long()
    x = s[name][pages].view(FP8).double() if codes is None else codes[pages]
    x = x * (s[name + "_scale"] if scales is None else scales)[pages].double()[:, :, None, None]
    if name == "v":
        x = x.transpose(2, 3)
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _exact_attention(s, q, held):
    c = s["case"]
    G, at = c["heads"] // c["kv_heads"], 0
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    for b, (n, m) in enumerate(zip(s["new"], s["total"])):
        k, v = (_exact_heads(s, name, b, *held.get(name, ())) for name in ("k", "v"))
        i, j = torch.arange(m - n, m, device=DEV)[:, None], torch.arange(m, device=DEV)
        see = (j <= i) if c["causal"] else torch.ones((n, m), dtype=torch.bool, device=DEV)
        if c["window"]:
            see = see & (j > i - c["window"])
        for h in range(c["heads"]):
            t = (q[at:at + n, h].double() @ k[h // G].T.contiguous()) * c["dim"] ** -0.5
            t = torch.where(see, t, -torch.inf)
            l = torch.logsumexp(t, -1, keepdim=True)
            out[at:at + n, h] = torch.exp(t - l) @ v[h // G]
            lse[at:at + n, h] = l[:, 0]
        at += n
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path == "rope":
        return {"q": _exact_rope(s, s["q"], s["wq"]), "k": _exact_rope(s, s["k_new"], s["wk"])}
    if path == "read":
        k, v = ([_exact_heads(s, n, b).transpose(0, 1) for b in range(case["batch"])] for n in ("k", "v"))
        return {"k_back": torch.cat(k), "v_back": torch.cat(v)}
    dt = DTYPES[case["dtype"]]
    q, k = s.get("q"), s["k_new"] if path == "write" else None
    if path == "step":
        q = _exact_rope(s, s["q"], s["wq"]).to(dt)
        k = _exact_rope(s, s["k_new"], s["wk"]).to(dt)
    held, got = {}, {}
    if path in ("write", "step"):
        held = {"k": _exact_write(s, "k", k), "v": _exact_write(s, "v", s["v_new"])}
        got = {"k": held["k"][0], "v": held["v"][0], "k_scale": held["k"][1], "v_scale": held["v"][1]}
        if path == "write":
            if case["back"]:
                for name in ("k", "v"):
                    rows = [_exact_heads(s, name, b, *held[name])[:, -s["new"][b]:].transpose(0, 1) for b in range(case["batch"])]
                    got[name + "_back"] = torch.cat(rows)
            return got
    out, lse = _exact_attention(s, q, held)
    return {**got, "out": out, "lse": lse}
