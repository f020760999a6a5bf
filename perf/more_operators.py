"""Rotary positions and an 8-bit paged key-value cache in a serving step's attention, as cases that can be timed and compared.

A step of an engine whose cache holds a byte per number and whose positions are rotations runs three operators, and a
program without a cache, or a backward pass, the rotation alone:
  * rotary: every head's vector turned by its token's position, in pairs of dimensions, over the whole head or a part of
    it, with frequencies as they are or stretched for long contexts; turned back for gradients;
  * append: the new tokens' keys, turned by their positions, and their values into the slots of a 16-bit paged cache; the
    queries are turned in the same call;
  * append8: the same into a cache of 8-bit floats with one scale per block of tokens and head. A scale is the least power
    of two s with amax <= 448 s over what its block holds; where new tokens let it grow, the block's older codes are
    divided by the growth and rounded again;
  * attn8: each new token against its request's keys and values in that cache through the block table.

The sizes are those of the repository's search spaces: up to 8192 sequences and 65536 tokens in a step, blocks of 8, 16 and
32 tokens, prompts up to 2560 tokens and sequences up to 8192, and longer ones for the split over a long cache.
exact() is in 64 bits; codes are returned as the 8-bit floats that they are, beside their scales.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
F8 = torch.float8_e4m3fn


def listed():
    return [
        # the queries of a decode step, each at its own sequence's length
        {"name": "rotary-decode", "op": "rotary", "dtype": "bf16", "D": 128, "rot": 128, "H": 32, "pairs": "half", "T": 251,
         "far": 2560, "stretch": "none", "back": False},
        # gradients of long prompts' queries: part of the head, neighbouring dimensions, a context stretched eight times
        {"name": "rotary-back", "op": "rotary", "dtype": "fp16", "D": 64, "rot": 32, "H": 28, "pairs": "interleaved", "T": 32767,
         "far": 131072, "stretch": "parts", "back": True},
        # a token per request: queries, keys and values of one layer
        {"name": "append-decode", "op": "append", "dtype": "bf16", "D": 128, "rot": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "pairs": "half", "stretch": "none", "dec": 251, "c_lo": 1, "c_hi": 2560, "pre": 0, "pad": 5},
        # prompts that spend half of the largest token budget, in a stretched context
        {"name": "append-budget", "op": "append", "dtype": "fp16", "D": 128, "rot": 128, "Hq": 28, "Hkv": 4, "bs": 32, "layout": "hnd",
         "pairs": "half", "stretch": "linear", "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 16, "q_lo": 1, "q_hi": 4001, "p_lo": 0,
         "p_hi": 60000, "pad": 0},
        # a token per request into blocks that mostly hold some already
        {"name": "append8-decode", "op": "append8", "dtype": "bf16", "D": 128, "rot": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "pairs": "half", "stretch": "none", "dec": 256, "c_lo": 1, "c_hi": 2560, "pre": 0, "pad": 0},
        # decodes and chunks together, part of the head rotated
        {"name": "append8-mixed", "op": "append8", "dtype": "fp16", "D": 64, "rot": 32, "Hq": 12, "Hkv": 12, "bs": 8, "layout": "hnd",
         "pairs": "interleaved", "stretch": "base", "dec": 190, "c_lo": 1, "c_hi": 2560, "pre": 5, "q_lo": 100, "q_hi": 640,
         "p_lo": 0, "p_hi": 1500, "pad": 3},
        # prompts that spend half of the largest token budget
        {"name": "append8-budget", "op": "append8", "dtype": "bf16", "D": 128, "rot": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "pairs": "half", "stretch": "none", "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 16, "q_lo": 1, "q_hi": 4001, "p_lo": 0, "p_hi": 0,
         "pad": 0},
        # a single user's next token: latency
        {"name": "attn8-one", "op": "attn8", "dtype": "bf16", "D": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 1, "c_lo": 776, "c_hi": 777, "pre": 0},
        # the decode step of the default number of sequences, ragged lengths up to the longest prompt
        {"name": "attn8-decode", "op": "attn8", "dtype": "bf16", "D": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 256, "c_lo": 64, "c_hi": 2560, "pre": 0},
        # a few very long sequences, seven query heads to a shared one: the long axis has to be split
        {"name": "attn8-long", "op": "attn8", "dtype": "fp16", "D": 128, "Hq": 28, "Hkv": 4, "bs": 32, "layout": "hnd",
         "dec": 3, "c_lo": 20000, "c_hi": 65535, "pre": 0},
        # chunked prefill under a token budget of about 2048: decodes and chunks in one batch, no shared heads, a window
        {"name": "attn8-mixed", "op": "attn8", "dtype": "fp16", "D": 64, "Hq": 12, "Hkv": 12, "bs": 8, "layout": "nhd",
         "dec": 190, "c_lo": 1, "c_hi": 2560, "pre": 5, "q_lo": 100, "q_hi": 640, "p_lo": 0, "p_hi": 1500, "window": 1024},
        # a chunk of a long prompt over what is cached of it: the tensor cores' rate is what counts
        {"name": "attn8-chunk", "op": "attn8", "dtype": "bf16", "D": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 1, "q_lo": 4096, "q_hi": 4096, "p_lo": 8192, "p_hi": 8192},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def _draw(rng):
    op = rng.choice(("rotary", "append", "append8", "append8", "attn8", "attn8", "attn8"))
    c = {"op": op, "dtype": rng.choice(("bf16", "fp16")), "D": rng.choice((64, 128, 80, 256) if op == "rotary" else (64, 128))}
    if op != "attn8":
        c.update(rot=rng.choice((c["D"], c["D"], 16, 32, 48)), pairs=rng.choice(("half", "interleaved")),
                 stretch=rng.choice(("none", "linear", "base", "parts")))
    if op == "rotary":
        c.update(H=rng.choice((1, 5, 8, 28, 32)), T=_log_int(rng, 1, 40000),
                 far=_log_int(rng, 16, 1 << 20), back=rng.random() < 0.3)
        return c
    c.update(bs=rng.choice((8, 16, 32)), layout=rng.choice(("nhd", "hnd")), Hkv=rng.choice((1, 2, 4, 5, 8)))
    c["Hq"] = c["Hkv"] * rng.choice((1, 2, 3, 4, 7, 8) if c["Hkv"] < 8 else (1, 2, 4))
    form = rng.choice(("decode", "chunk", "mixed"))
    c.update(dec=0, c_lo=1, c_hi=1, pre=0, q_lo=1, q_hi=1, p_lo=0, p_hi=0)
    if op != "attn8":
        c["pad"] = rng.choice((0, 0, 1, 13))
        if form != "chunk":
            c.update(dec=_log_int(rng, 2, 4096), c_lo=1, c_hi=_log_int(rng, 16, 8192))
        if form != "decode":
            c.update(pre=rng.randint(1, 8), q_lo=1, q_hi=_log_int(rng, 32, 4000), p_lo=0, p_hi=_log_int(rng, 1, 100000))
        return c
    if form == "decode":
        # few sequences may be long ones
        n = _log_int(rng, 1, 256)
        hi = _log_int(rng, 64, max(2560, 65536 // n))
        c.update(dec=n, c_lo=max(1, hi // rng.choice((2, 8, 64))), c_hi=hi)
    elif form == "chunk":
        c.update(pre=rng.randint(1, 4), q_lo=1, q_hi=_log_int(rng, 4, 2500), p_lo=0, p_hi=_log_int(rng, 1, 8192))
    else:
        c.update(dec=_log_int(rng, 4, 200), c_lo=1, c_hi=_log_int(rng, 64, 2560), pre=rng.randint(1, 5), q_lo=2,
                 q_hi=_log_int(rng, 16, 700), p_lo=0, p_hi=_log_int(rng, 1, 1500))
    mask = rng.random()
    if mask < 0.25:
        c["window"] = _log_int(rng, 16, 2048)
    elif mask < 0.35:
        c["causal"] = False
    return c


# ---------------------------------------------------------------------------------------------- lengths and places

def _spread(n, lo, hi, step):
    """n integers spread evenly over lo .. hi, in no order."""
    return [lo + int((hi - lo + 1) * (((i + 0.5) * step) % 1.0)) for i in range(n)]


def _requests(case):
    """[(tokens in the cache, new tokens)] of the batch's requests, decodes first."""
    gold = 0.6180339887498949
    out = [(c, 1) for c in _spread(case["dec"], case["c_lo"], case["c_hi"], gold)]
    if case["pre"]:
        out += list(zip(_spread(case["pre"], case["p_lo"], case["p_hi"], 0.7548776662466927),
                        _spread(case["pre"], case["q_lo"], case["q_hi"], gold)))
    return out


def _blocks(n, bs):
    return (n + bs - 1) // bs


def _batch(case, seed):
    """(lengths in the batch's order: cached, new)"""
    rng = np.random.default_rng(seed * 16 + 3)
    req = [_requests(case)[i] for i in rng.permutation(case["dec"] + case["pre"])]
    return rng, np.array([r[0] for r in req], np.int64), np.array([r[1] for r in req], np.int64)


def _places(case, seed):
    """Position and cache slot of each token of an append, requests back to back, then padded tokens without a slot; the
    number of blocks. Only the blocks that the new tokens touch are in the cache, anywhere in it."""
    rng, cached, new = _batch(case, seed)
    bs = case["bs"]
    first = cached // bs
    count = _blocks(cached + new, bs) - first
    n_blocks = int(count.sum()) + 3
    ids, base = rng.permutation(n_blocks), np.cumsum(count) - count
    r = np.repeat(np.arange(len(new)), new)
    p = cached[r] + np.arange(len(r)) - (np.cumsum(new) - new)[r]
    slot = ids[base[r] + p // bs - first[r]] * bs + p % bs
    pad = case["pad"]
    return np.concatenate([p, np.zeros(pad, np.int64)]).astype(np.int32), np.concatenate([slot, np.full(pad, -1)]).astype(np.int64), n_blocks


def _cache_of(case, seed):
    """What an attention reads through: lengths, the block table (blocks anywhere in the cache), the number of blocks."""
    rng, cached, new = _batch(case, seed)
    count = _blocks(cached + new, case["bs"])
    n_blocks = int(count.sum()) + 3
    ids, base = rng.permutation(n_blocks).astype(np.int32), np.cumsum(count) - count
    j = np.arange(int(count.max()))[None, :]
    table = np.where(j < count[:, None], ids[np.minimum(base[:, None] + j, n_blocks - 1)], -1).astype(np.int32)
    return {"cached": cached, "new": new, "table": table, "n_blocks": n_blocks, "T": int(new.sum())}


STRETCH = {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 4.0},
           "parts": {"factor": 8.0, "low": 1.0, "high": 32.0, "original_len": 8192}}


def _magnitude(case):
    return 0.1 * math.log(8.0) + 1.0 if case["stretch"] == "parts" else 1.0


def _frequencies(case):
    """Radians per position of each pair of dimensions."""
    d, s, how = case["rot"], STRETCH[case["stretch"]], case["stretch"]
    base = 10000.0 * (s["factor"] ** (d / (d - 2)) if how == "base" else 1.0)
    f = base ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    if how == "linear":
        f = f / s["factor"]
    if how == "parts":   # what turns often in the original context stays, what turns less than once is slowed
        keep = np.clip((s["original_len"] * f / (2 * np.pi) - s["low"]) / (s["high"] - s["low"]), 0.0, 1.0)
        f = f * keep + f / s["factor"] * (1.0 - keep)
    return f


# ---------------------------------------------------------------------------------------------- inputs

def _normal(shape, dtype, gen, spread=None):
    t = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)
    return (t if spread is None else t.mul_(spread)).to(dtype)


def _shape(case, n_blocks):
    return (n_blocks, case["bs"], case["Hkv"], case["D"]) if case["layout"] == "nhd" else (n_blocks, case["Hkv"], case["bs"], case["D"])


def _tokens(case, x):
    """[block][token][head][dim] of a cache laid out either way."""
    return x if case["layout"] == "nhd" else x.transpose(1, 2)


def _power(e):
    """2^e of whole exponents, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _least_scale(amax):
    """The least power of two s with amax <= 448 s, at least 2^-100."""
    m, e = torch.frexp(amax)   # 448 = 0.875 * 2^9
    return _power(torch.where(m > 0.875, e - 8, e - 9).int().clamp(min=-100))


def _coded(case, n_blocks, gen, outlier):
    """A cache of 8-bit floats with a scale per block and head; some dimensions of keys are larger than the others."""
    spread = torch.ones(case["D"], device="cuda")
    spread[:: 16] = outlier
    x = _normal(_shape(case, n_blocks), torch.float32, gen, spread)
    s = _least_scale(x.abs().amax((1, 3) if case["layout"] == "nhd" else (2, 3)))
    codes = (x / (s[:, None, :, None] if case["layout"] == "nhd" else s[:, :, None, None])).to(F8)
    return _tokens(case, codes), s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 16 + 5)
    op, dt, D = case["op"], DTYPES[case["dtype"]], case["D"]

    def dev(a, dtype=torch.int32):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)

    st = {"case": case}
    if op == "rotary":
        st["x"] = _normal((case["T"], case["H"], D), dt, gen)
        st["out"] = torch.empty_like(st["x"])
        st["position"] = dev(np.random.default_rng(seed * 16 + 3).integers(0, case["far"], case["T"]))
    elif op == "attn8":
        st["h"] = h = _cache_of(case, seed)
        st["k_cache"], st["k_scale"] = _coded(case, h["n_blocks"], gen, 4.0)
        st["v_cache"], st["v_scale"] = _coded(case, h["n_blocks"], gen, 1.0)
        st["q"] = _normal((h["T"], case["Hq"], D), dt, gen)
        st["table"], st["kv_len"] = dev(h["table"]), dev(h["cached"] + h["new"])
        st["query_start"] = dev(np.concatenate([[0], np.cumsum(h["new"])]))
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
        st["scale"], st["most"] = 1.0 / math.sqrt(D), int(h["new"].max())
    else:
        position, slot, n_blocks = _places(case, seed)
        st["position"], st["slot"] = dev(position), dev(slot, torch.int64)
        # a projection's output holds a token's queries, keys and values side by side
        qkv = _normal((len(slot), case["Hq"] + 2 * case["Hkv"], D), dt, gen)
        st["q"], st["k"], st["v"] = qkv.split((case["Hq"], case["Hkv"], case["Hkv"]), 1)
        st["q_out"] = torch.zeros((len(slot), case["Hq"], D), dtype=dt, device="cuda")
        if op == "append8":
            # what the blocks held before came of smaller numbers: most scales grow by the first pass
            st["k_cache"], st["k_scale"] = _coded(case, n_blocks, gen, 0.25)
            st["v_cache"], st["v_scale"] = _coded(case, n_blocks, gen, 0.25)
        else:
            st["k_cache"], st["v_cache"] = (_tokens(case, _normal(_shape(case, n_blocks), dt, gen)) for _ in range(2))
    if op != "attn8":
        st["frequencies"], st["magnitude"] = dev(_frequencies(case), torch.float64), _magnitude(case)
    if own:
        from paper_2408_04323_gb300 import scoot as S
        st["S"], st["ctx"] = S, S.Context(torch.cuda.current_device())
        if op != "attn8":
            st["rotation"] = S.Rotation(case["rot"], base=10000.0, interleaved=case["pairs"] == "interleaved", stretch=case["stretch"],
                                        magnitude=st["magnitude"], **STRETCH[case["stretch"]])
    return st


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    op = st["case"]["op"]
    if own:
        return {"rotary": _own_rotary, "append": _own_append, "append8": _own_append8, "attn8": _own_attn8}[op](st)
    return {"rotary": _plain_rotary, "append": _plain_append, "append8": _plain_append8, "attn8": _plain_attn8}[op](st)


def _own_rotary(st):
    st["S"].scoot_rotary(st["ctx"], st["rotation"], st["x"], st["position"], st["out"], inverse=st["case"]["back"])
    return st["out"]


def _own_append(st):
    st["S"].scoot_kv_append_rotary(st["ctx"], st["rotation"], st["k"], st["v"], st["slot"], st["position"], st["k_cache"], st["v_cache"],
                                   q=st["q"], q_out=st["q_out"])
    return st["q_out"], st["k_cache"], st["v_cache"]


def _own_append8(st):
    st["S"].scoot_kv_append8(st["ctx"], st["k"], st["v"], st["slot"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"],
                             rotation=st["rotation"], position=st["position"], q=st["q"], q_out=st["q_out"])
    return st["q_out"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"]


def _own_attn8(st):
    c = st["case"]
    st["S"].scoot_paged_attention8(st["ctx"], st["q"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["table"],
                                   st["query_start"], st["kv_len"], st["out"], scale=st["scale"], causal=c.get("causal", True),
                                   window=c.get("window", 0), lse=st["lse"], max_new=st["most"])
    return st["out"], st["lse"]


def _turned(st, x, position, back=False):
    """x [token][head][dim] in 32 bits, its pairs of dimensions turned by position * frequency."""
    rot, half = st["case"]["rot"], st["case"]["rot"] // 2
    angle = position.double()[:, None] * st["frequencies"] * (-1.0 if back else 1.0)
    cos, sin = (f(angle).float()[:, None, :] * st["magnitude"] for f in (torch.cos, torch.sin))
    x, y = x.float(), x.float().clone()
    if st["case"]["pairs"] == "half":
        a, b = x[..., :half], x[..., half:rot]
        y[..., :half], y[..., half:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_rotary(st):
    st["out"].copy_(_turned(st, st["x"], st["position"], st["case"]["back"]))
    return st["out"]


def _plain_append(st):
    bs = st["case"]["bs"]
    there = torch.nonzero(st["slot"] >= 0)[:, 0]   # padded tokens have none
    slot, position = st["slot"][there], st["position"][there]
    st["q_out"][there] = _turned(st, st["q"][there], position).to(st["q"].dtype)
    st["k_cache"][slot // bs, slot % bs] = _turned(st, st["k"][there], position).to(st["k"].dtype)
    st["v_cache"][slot // bs, slot % bs] = st["v"][there]
    return st["q_out"], st["k_cache"], st["v_cache"]


def _plain_append8(st):
    bs = st["case"]["bs"]
    there = torch.nonzero(st["slot"] >= 0)[:, 0]
    slot, position = st["slot"][there], st["position"][there]
    st["q_out"][there] = _turned(st, st["q"][there], position).to(st["q"].dtype)
    _plain_coded(st["k_cache"], st["k_scale"], _turned(st, st["k"][there], position), slot // bs, slot % bs)
    _plain_coded(st["v_cache"], st["v_scale"], st["v"][there].float(), slot // bs, slot % bs)
    return st["q_out"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"]


def _plain_coded(cache, scale, x, block, at):
    """x [token][head][dim] into the blocks: a block keeps its scale if it held tokens and they and the new ones fit it."""
    bs, held = cache.shape[1], cache.view(torch.uint8)
    amax = torch.zeros_like(scale).index_reduce_(0, block, x.abs().amax(-1), "amax")
    first = torch.full((len(scale),), bs, device="cuda").scatter_reduce_(0, block, at, "amin")   # of the new ones
    new = torch.where((first > 0)[:, None], torch.maximum(_least_scale(amax), scale), _least_scale(amax))
    new = torch.where((first < bs)[:, None], new, scale)
    grown = torch.nonzero((first > 0) & (first < bs) & (new > scale).any(1))[:, 0]
    old = held[grown].view(F8).float() * (scale[grown] / new[grown])[:, None, :, None]
    older = torch.arange(bs, device="cuda") < first[grown, None]
    held[grown] = torch.where(older[:, :, None, None], old.to(F8).view(torch.uint8), held[grown])
    scale.copy_(new)
    held[block, at] = (x / new[block][:, :, None]).to(F8).view(torch.uint8)


def _plain_attn8(st):
    # requests with one new token, and those with more: each kind padded to its longest
    new = st["h"]["new"]
    _plain_padded(st, np.flatnonzero(new == 1))
    _plain_padded(st, np.flatnonzero(new > 1))
    return st["out"], st["lse"]


def _plain_padded(st, rows):
    if not len(rows):
        return
    c, h = st["case"], st["h"]
    bs, D, Hq, Hkv = c["bs"], c["D"], c["Hq"], c["Hkv"]
    window, causal = c.get("window", 0), c.get("causal", True)
    n, most = int(h["new"][rows].max()), _blocks(int((h["cached"] + h["new"])[rows].max()), bs)
    r = torch.from_numpy(rows).cuda()
    ids = st["table"][r, :most].long().clamp(min=0)
    K, V = ((cache.view(torch.uint8)[ids].view(F8).float() * scale[ids][:, :, None, :, None]).flatten(1, 2).permute(0, 2, 3, 1)
            for cache, scale in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])))   # [R][Hkv][D][keys]
    total, start = st["kv_len"][r].long(), st["query_start"][r].long()
    count = st["query_start"][r + 1].long() - start
    j = torch.arange(n, device="cuda")
    live = j < count[:, None]
    token = torch.where(live, start[:, None] + j, 0)                                             # [R][n]
    q = st["q"][token].float().reshape(len(rows), n, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.flatten(2, 3), K).unflatten(2, (Hq // Hkv, n)).mul_(st["scale"])          # [R][Hkv][G][n][keys]
    key, position = torch.arange(most * bs, device="cuda"), (total - count)[:, None] + j
    seen = (key < total[:, None])[:, None] & ((key <= position[..., None]) if causal else live[..., None])
    if window:
        seen = seen & (key > position[..., None] - window)
    s.masked_fill_(~seen[:, None, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), V.transpose(2, 3)).unflatten(2, (Hq // Hkv, n)) / z
    at = torch.nonzero(live)
    st["out"][token[live]] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[at[:, 0], at[:, 1]].to(st["out"].dtype)
    st["lse"][token[live]] = (m + torch.log(z))[..., 0].permute(0, 3, 1, 2).flatten(2, 3)[at[:, 0], at[:, 1]]


# ---------------------------------------------------------------------------------------------- floors

def _seen(case):
    """(pairs of a new token and a key that it sees, keys that some token of their request sees)."""
    window, causal = case.get("window", 0), case.get("causal", True)
    pairs = keys = 0
    for cached, n in _requests(case):
        pos = np.arange(cached, cached + n, dtype=np.int64)
        last = pos + 1 if causal else np.full(n, cached + n, dtype=np.int64)
        first = np.maximum(pos + 1 - window, 0) if window else np.zeros(n, np.int64)
        pairs += int((last - first).sum())
        keys += cached + n - int(first[0])
    return pairs, keys


def work(case):
    D = case["D"]
    if case["op"] == "rotary":
        n = case["T"] * case["H"]
        return {"bytes": 2 * 2 * n * D + 4 * case["T"], "flops": 3 * n * case["rot"]}
    req, bs, Hq, Hkv = _requests(case), case["bs"], case["Hq"], case["Hkv"]
    T = sum(n for _, n in req)
    if case["op"] == "append":
        return {"bytes": 2 * 2 * T * (Hq + 2 * Hkv) * D + 12 * T, "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    if case["op"] == "append8":
        # two bytes in and one out of each key and value, two and two of a query; scales out, those of begun blocks in
        scales = 8 * Hkv * sum(_blocks(c + n, bs) - c // bs + (c % bs > 0) for c, n in req)
        return {"bytes": T * (2 * 2 * Hq + 3 * 2 * Hkv) * D + 12 * T + scales, "flops": 3 * T * (Hq + Hkv) * case["rot"] + 4 * T * Hkv * D}
    pairs, keys = _seen(case)
    blocks = sum(_blocks(c + n, bs) for c, n in req)
    return {"bytes": 2 * 2 * T * Hq * D + 4 * T * Hq + 2 * keys * Hkv * D + 8 * (keys // bs) * Hkv + 4 * blocks + 8 * len(req),
            "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    op = case["op"]
    if op == "attn8":
        return _exact_attention(case, seed)
    st = prepare(case, seed)
    rot = case["rot"]
    pos = st["position"].double()
    if op == "rotary" and case["back"]:
        pos = -pos
    turn = torch.polar(torch.full((len(pos), rot // 2), st["magnitude"], dtype=torch.float64, device="cuda"),
                       torch.outer(pos, torch.from_numpy(_frequencies(case)).cuda()))

    def turned(x):
        part = x[..., :rot].double()
        z = torch.complex(*(part.chunk(2, -1) if case["pairs"] == "half" else (part[..., 0::2], part[..., 1::2]))) * turn[:, None, :]
        z = torch.cat([z.real, z.imag], -1) if case["pairs"] == "half" else torch.view_as_real(z).flatten(-2)
        return torch.cat([z, x[..., rot:].double()], -1)

    if op == "rotary":
        return turned(st["x"])
    there = st["slot"] >= 0
    q = st["q_out"].double()
    q[there] = turned(st["q"])[there]
    slot = st["slot"][there]
    if op == "append":
        k, v = st["k_cache"].double(), st["v_cache"].double()
        k[slot // case["bs"], slot % case["bs"]] = turned(st["k"])[there]
        v[slot // case["bs"], slot % case["bs"]] = st["v"][there].double()
        return q, k, v
    out = []
    for cache, scale, x in ((st["k_cache"], st["k_scale"], turned(st["k"])[there]), (st["v_cache"], st["v_scale"], st["v"][there].double())):
        # what a block holds, in units of its scale, before any rounding: the older tokens' numbers and the new ones'
        held, bs = cache.double(), case["bs"]
        value = held * scale.double()[:, None, :, None]
        old = torch.zeros(held.shape[:2], dtype=torch.bool, device="cuda")
        new = torch.zeros_like(old)
        b, a = slot // bs, slot % bs
        new[b, a] = True
        begin = torch.where(new.any(1), new.int().argmax(1), bs)
        old = (torch.arange(bs, device="cuda") < begin[:, None]) & new.any(1)[:, None]
        value[b, a] = x
        top = (x.new_zeros(held.shape[:3])).index_put_((b, a), x.abs().amax(-1)).amax(1)
        need = torch.exp2(torch.ceil(torch.log2(top / 448.0))).clamp(min=2.0 ** -100)
        kept = (begin > 0)[:, None] & (scale.double() > need)
        s = torch.where(new.any(1)[:, None], torch.where(kept, scale.double(), need), scale.double())
        out.append((torch.where((old | new)[:, :, None, None], value / s[:, None, :, None], held), s))
    return q, out[0][0], out[1][0], out[0][1], out[1][1]


def _exact_attention(case, seed):
    if 4 * case["D"] * case["Hq"] * _seen(case)[0] > 4e12:
        return None
    st = prepare(case, seed)
    h, bs, D, Hkv = st["h"], case["bs"], case["D"], case["Hkv"]
    G = case["Hq"] // Hkv
    window, causal = case.get("window", 0), case.get("causal", True)
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    begin = np.concatenate([[0], np.cumsum(h["new"])])
    for r in range(len(h["new"])):
        n, total = int(h["new"][r]), int(h["cached"][r] + h["new"][r])
        ids = torch.from_numpy(h["table"][r, :_blocks(total, bs)].astype(np.int64)).cuda()
        K, V = ((c.view(torch.uint8)[ids].view(F8).double() * s[ids].double()[:, None, :, None]).reshape(-1, Hkv, D)[:total]
                for c, s in ((st["k_cache"], st["k_scale"]), (st["v_cache"], st["v_scale"])))
        step = max(1, (1 << 26) // (total * case["Hq"]))
        for a in range(0, n, step):
            b = min(n, a + step)
            p = torch.arange(total - n + a, total - n + b, device="cuda")[:, None]
            i = torch.arange(total, device="cuda")[None, :]
            hidden = torch.zeros((b - a, total), dtype=torch.bool, device="cuda")
            if causal:
                hidden |= i > p
            if window:
                hidden |= i <= p - window
            at = slice(int(begin[r]) + a, int(begin[r]) + b)
            q = st["q"][at].double().unflatten(1, (Hkv, G))
            s = (torch.einsum("tcgd,kcd->tcgk", q, K) * st["scale"]).masked_fill(hidden[:, None, None, :], -math.inf)
            z = torch.logsumexp(s, -1)
            out[at] = torch.einsum("tcgk,kcd->tcgd", torch.exp(s - z[..., None]), V).flatten(1, 2)
            lse[at] = z.flatten(1, 2)
    return out, lse
