"""The attention part of a serving step over a paged key-value cache, as cases that can be timed and compared.

The parameters that a tuner of an inference engine searches (most sequences and most batched tokens of a step, the
cache's block size, chunked prefill) act on three operators, which a step runs in this order:
  * tables: from the lengths of the requests, the blocks that their new tokens take from the free ones, each request's
    row of the block table, and the position and cache slot of every new token;
  * append: the new tokens' keys and values into those slots;
  * attn: each new token against its request's keys and values through the block table: a chunk of a prompt, a single
    token per request, or both in one batch; causal, over a window, or over the whole cache.

The sizes are those of the repository's search spaces: up to 8192 sequences and 65536 tokens in a step, blocks of 8, 16 and
32 tokens, prompts up to 2560 tokens and sequences up to 8192, and longer ones for the split over a long cache.
exact() is plain numpy and torch in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_ROWS = 1 << 25   # scores that the plain form holds at a time


def listed():
    return [
        # a step of a lightly loaded engine: every request decodes one token; latency is what counts
        {"name": "tables-decode", "op": "tables", "bs": 16, "dec": 48, "c_lo": 1, "c_hi": 2560, "pre": 0},
        # an ordinary step of chunked prefill: decodes, and a few prompts' chunks that share the token budget
        {"name": "tables-mixed", "op": "tables", "bs": 32, "dec": 249, "c_lo": 1, "c_hi": 2560, "pre": 7,
         "q_lo": 33, "q_hi": 1023, "p_lo": 0, "p_hi": 2047},
        # the most sequences, and nearly the most tokens, of the search space, in its smallest blocks
        {"name": "tables-wide", "op": "tables", "bs": 8, "dec": 8064, "c_lo": 1, "c_hi": 2560, "pre": 128,
         "q_lo": 1, "q_hi": 896, "p_lo": 0, "p_hi": 1024},
        # the keys and values of one token per request
        {"name": "append-decode", "op": "append", "dtype": "bf16", "D": 128, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 251, "c_lo": 1, "c_hi": 2560, "pre": 0},
        # one prompt's chunk, heads outside the block's tokens
        {"name": "append-chunk", "op": "append", "dtype": "fp16", "D": 64, "Hkv": 4, "bs": 32, "layout": "hnd",
         "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 3, "q_lo": 2049, "q_hi": 4095, "p_lo": 0, "p_hi": 1000},
        # a step that spends the largest token budget
        {"name": "append-budget", "op": "append", "dtype": "bf16", "D": 128, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 32, "q_lo": 1, "q_hi": 3985, "p_lo": 0, "p_hi": 0},
        # a single user's next token: latency
        {"name": "attn-one", "op": "attn", "dtype": "bf16", "D": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 1, "c_lo": 776, "c_hi": 777, "pre": 0},
        # the decode step of the default number of sequences, ragged lengths up to the longest prompt
        {"name": "attn-decode", "op": "attn", "dtype": "bf16", "D": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 256, "c_lo": 64, "c_hi": 2560, "pre": 0},
        # a few very long sequences, seven query heads to a shared one: the long axis has to be split
        {"name": "attn-long", "op": "attn", "dtype": "fp16", "D": 128, "Hq": 28, "Hkv": 4, "bs": 32, "layout": "hnd",
         "dec": 3, "c_lo": 20000, "c_hi": 65535, "pre": 0},
        # chunked prefill under a token budget of about 2048: decodes and chunks in one batch, no shared heads
        {"name": "attn-mixed", "op": "attn", "dtype": "bf16", "D": 64, "Hq": 12, "Hkv": 12, "bs": 8, "layout": "nhd",
         "dec": 190, "c_lo": 1, "c_hi": 2560, "pre": 5, "q_lo": 100, "q_hi": 640, "p_lo": 0, "p_hi": 1500},
        # a chunk of a long prompt over what is cached of it: the tensor cores' rate is what counts
        {"name": "attn-chunk", "op": "attn", "dtype": "bf16", "D": 128, "Hq": 32, "Hkv": 8, "bs": 16, "layout": "nhd",
         "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 1, "q_lo": 8192, "q_hi": 8192, "p_lo": 8192, "p_hi": 8192},
        # prompts of odd lengths whose tokens see the last 1024 positions
        {"name": "attn-window", "op": "attn", "dtype": "fp16", "D": 64, "Hq": 14, "Hkv": 2, "bs": 16, "layout": "nhd",
         "dec": 0, "c_lo": 1, "c_hi": 1, "pre": 4, "q_lo": 1801, "q_hi": 2047, "p_lo": 0, "p_hi": 777, "window": 1024},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "append", "append", "attn", "attn", "attn", "attn"))
    c = {"op": op, "bs": rng.choice((8, 16, 32))}
    form = rng.choice(("decode", "chunk", "mixed"))
    c.update(dec=0, c_lo=1, c_hi=1, pre=0, q_lo=1, q_hi=1, p_lo=0, p_hi=0)
    if op == "tables":
        if form != "chunk":
            c.update(dec=_log_int(rng, 1, 8064), c_lo=1, c_hi=_log_int(rng, 16, 2560))
        if form != "decode":
            c.update(pre=_log_int(rng, 1, 128), q_lo=1, q_hi=_log_int(rng, 2, 896), p_lo=0, p_hi=_log_int(rng, 1, 1024))
        return c
    c.update(dtype=rng.choice(("bf16", "fp16")), D=rng.choice((64, 128)), layout=rng.choice(("nhd", "hnd")))
    if op == "append":
        c["Hkv"] = rng.choice((1, 2, 4, 5, 8))
        if form != "chunk":
            c.update(dec=_log_int(rng, 2, 4096), c_lo=1, c_hi=_log_int(rng, 16, 512))
        if form != "decode":
            c.update(pre=rng.randint(1, 8), q_lo=1, q_hi=_log_int(rng, 32, 6000), p_lo=0, p_hi=_log_int(rng, 1, 2000))
        return c
    c["Hkv"] = rng.choice((1, 2, 4, 8))
    c["Hq"] = c["Hkv"] * rng.choice((1, 2, 3, 4, 7, 8) if c["Hkv"] < 8 else (1, 2, 4))
    if form == "decode":
        # few sequences may be long ones
        n = _log_int(rng, 1, 256)
        hi = _log_int(rng, 64, max(2560, 65536 // n))
        c.update(dec=n, c_lo=max(1, hi // rng.choice((2, 8, 64))), c_hi=hi)
    elif form == "chunk":
        c.update(pre=rng.randint(1, 4), q_lo=1, q_hi=_log_int(rng, 4, 3500), p_lo=0, p_hi=_log_int(rng, 1, 8192))
    else:
        c.update(dec=_log_int(rng, 4, 200), c_lo=1, c_hi=_log_int(rng, 64, 2560), pre=rng.randint(1, 5), q_lo=8,
                 q_hi=_log_int(rng, 16, 700), p_lo=0, p_hi=_log_int(rng, 1, 1500))
    mask = rng.random()
    if mask < 0.25:
        c["window"] = _log_int(rng, 16, 2048)
    elif mask < 0.35:
        c["causal"] = False
    return c


# ---------------------------------------------------------------------------------------------- lengths

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


def _host(case, seed):
    """What the scheduler of an engine holds: lengths in the batch's order, the block table as the cached tokens left it,
    and the free blocks.  Blocks of a request lie anywhere in the cache."""
    rng = np.random.default_rng(seed * 16 + 3)
    req = [_requests(case)[i] for i in rng.permutation(case["dec"] + case["pre"])]
    bs = case["bs"]
    cached, new = (np.array([r[j] for r in req], np.int32) for j in (0, 1))
    held, full = _blocks(cached, bs), _blocks(cached + new, bs)
    take = int((full - held).sum())
    spare = 3 + take // 8
    n_blocks = int(held.sum()) + take + spare
    ids = rng.permutation(n_blocks).astype(np.int32)
    width = int(full.max())
    table = np.full((len(req), width), -1, np.int32)
    at = 0
    for r, h in enumerate(held):
        table[r, :h] = ids[at:at + h]
        at += h
    free = ids[at:].copy()
    return {"cached": cached, "new": new, "table": table, "free": free, "n_blocks": n_blocks, "T": int(new.sum())}


def _stepped(case, h):
    """The table after the new tokens' blocks were taken, and each new token's request, position and slot."""
    bs, table = case["bs"], h["table"].copy()
    at, request, position, slot = 0, [], [], []
    for r, (c, n) in enumerate(zip(h["cached"].tolist(), h["new"].tolist())):
        a, b = _blocks(c, bs), _blocks(c + n, bs)
        table[r, a:b] = h["free"][at:at + b - a]
        at += b - a
        p = np.arange(c, c + n)
        request.append(np.full(n, r))
        position.append(p)
        slot.append(table[r, p // bs].astype(np.int64) * bs + p % bs)
    cat = [np.concatenate(x) for x in (request, position, slot)]
    return table, at, cat[0], cat[1].astype(np.int32), cat[2].astype(np.int64)


# ---------------------------------------------------------------------------------------------- inputs

def _cache(case, n_blocks, gen):
    """Keys and values of a cache [block][token][head][dim]; "hnd" has the heads outside the tokens in memory."""
    Hkv, D, bs = case["Hkv"], case["D"], case["bs"]
    shape = (n_blocks, bs, Hkv, D) if case["layout"] == "nhd" else (n_blocks, Hkv, bs, D)
    out = []
    for _ in range(2):
        t = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=gen)
        out.append(t if case["layout"] == "nhd" else t.transpose(1, 2))
    return out


def prepare(case, seed):
    h = _host(case, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed * 16 + 5)

    def dev(a, dtype=torch.int32):
        return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)

    st = {"case": case, "h": h, "cached": dev(h["cached"]), "new": dev(h["new"]), "table": dev(h["table"]), "free": dev(h["free"])}
    R, T, op = len(h["new"]), h["T"], case["op"]
    if op == "tables":
        st["out"] = {"query_start": torch.empty(R + 1, dtype=torch.int32, device="cuda"),
                     "kv_len": torch.empty(R, dtype=torch.int32, device="cuda"),
                     "slot": torch.empty(T, dtype=torch.int64, device="cuda"),
                     "position": torch.empty(T, dtype=torch.int32, device="cuda"),
                     "counts": torch.empty(2, dtype=torch.int32, device="cuda")}
    else:
        table, _, request, position, slot = _stepped(case, h)
        st["k_cache"], st["v_cache"] = _cache(case, h["n_blocks"], gen)
        dt, D = DTYPES[case["dtype"]], case["D"]
        if op == "append":
            # a projection's output holds a token's keys and values side by side
            kv = torch.empty((T, 2, case["Hkv"], D), dtype=dt, device="cuda").normal_(generator=gen)
            st["k"], st["v"] = kv[:, 0], kv[:, 1]
            st["slot"] = dev(slot, torch.int64)
        else:
            st["q"] = torch.empty((T, case["Hq"], D), dtype=dt, device="cuda").normal_(generator=gen)
            st["table"] = dev(table)
            st["query_start"] = dev(np.concatenate([[0], np.cumsum(h["new"])]))
            st["kv_len"] = dev(h["cached"] + h["new"])
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty((T, case["Hq"]), dtype=torch.float32, device="cuda")
            st["scale"] = 1.0 / math.sqrt(D)
    if own:
        from paper_2408_04323_gb300 import scoot as S
        st["S"], st["ctx"] = S, S.Context(torch.cuda.current_device())
    return st


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    op = st["case"]["op"]
    if own:
        return {"tables": _own_tables, "append": _own_append, "attn": _own_attn}[op](st)
    return {"tables": _plain_tables, "append": _plain_append, "attn": _plain_attn}[op](st)


def _own_tables(st):
    o = st["out"]
    st["S"].scoot_kv_tables(st["ctx"], st["cached"], st["new"], st["table"], st["case"]["bs"], st["h"]["n_blocks"], st["free"],
                            o["query_start"], o["kv_len"], o["slot"], o["position"], o["counts"])
    return {"table": st["table"], **o}


def _own_append(st):
    st["S"].scoot_kv_append(st["ctx"], st["k"], st["v"], st["slot"], st["k_cache"], st["v_cache"])
    return st["k_cache"], st["v_cache"]


def _own_attn(st):
    c = st["case"]
    st["S"].scoot_paged_attention(st["ctx"], st["q"], st["k_cache"], st["v_cache"], st["table"], st["query_start"],
                                  st["kv_len"], st["out"], scale=st["scale"], causal=c.get("causal", True),
                                  window=c.get("window", 0), lse=st["lse"])
    return st["out"], st["lse"]


def _plain_tables(st):
    """A request takes the blocks that its new tokens need beyond those it holds, in the requests' order; one whose blocks
    the free ones do not cover is refused: it takes none, its tokens have no slot and it has nothing to attend to."""
    bs, T = st["case"]["bs"], st["h"]["T"]
    cached, new, table, free = st["cached"].long(), st["new"].long(), st["table"], st["free"]
    held = (cached + bs - 1) // bs
    need = (cached + new + bs - 1) // bs - held
    end = torch.cumsum(need, 0)
    fits = (need == 0) | (end <= free.numel())
    col = torch.arange(table.shape[1], device="cuda")
    fresh = (col >= held[:, None]) & (col < (held + need)[:, None]) & fits[:, None]
    which = ((end - need)[:, None] + col - held[:, None]).clamp(0, free.numel() - 1)
    table = torch.where(fresh, free[which], table)
    stop = torch.cumsum(new, 0)
    t = torch.arange(T, device="cuda")
    r = torch.searchsorted(stop, t, right=True)
    p = cached[r] + t - (stop - new)[r]
    slot = torch.where(fits[r], table[r, p // bs].long() * bs + p % bs, torch.full_like(p, -1))
    start = torch.cat([torch.zeros_like(stop[:1]), stop])
    counts = torch.stack([(need * fits).sum(), (~fits).sum()])
    return {"table": table, "query_start": start.int(), "kv_len": ((cached + new) * fits).int(), "slot": slot,
            "position": p.int(), "counts": counts.int()}


def _plain_append(st):
    bs = st["case"]["bs"]
    slot = st["slot"]
    st["k_cache"][slot // bs, slot % bs] = st["k"]
    st["v_cache"][slot // bs, slot % bs] = st["v"]
    return st["k_cache"], st["v_cache"]


def _plain_attn(st):
    c, h = st["case"], st["h"]
    bs, D, Hq, Hkv = c["bs"], c["D"], c["Hq"], c["Hkv"]
    window, causal = c.get("window", 0), c.get("causal", True)
    out, lse = torch.empty_like(st["q"]), torch.empty_like(st["lse"])
    at = 0
    for r, (cached, n) in enumerate(zip(h["cached"].tolist(), h["new"].tolist())):
        total = cached + n
        ids = st["table"][r, :_blocks(total, bs)].long()
        K, V = (x[ids].flatten(0, 1)[:total].float().permute(1, 0, 2) for x in (st["k_cache"], st["v_cache"]))  # [Hkv][total][D]
        step = max(1, _ROWS // (total * Hq))
        for a in range(0, n, step):
            b = min(n, a + step)
            q = st["q"][at + a:at + b].float().reshape(b - a, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3)
            s = torch.matmul(q.flatten(1, 2), K.transpose(1, 2)).reshape(Hkv, Hq // Hkv, b - a, total) * st["scale"]
            pos = torch.arange(cached + a, cached + b, device="cuda")[:, None]
            key = torch.arange(total, device="cuda")
            seen = key <= pos if causal else key >= 0
            if window:
                seen = seen & (key > pos - window)
            s = torch.where(seen, s, float("-inf"))
            m = s.amax(-1, keepdim=True)
            p = torch.exp(s - m)
            z = p.sum(-1, keepdim=True)
            o = torch.matmul(p.flatten(1, 2), V).reshape(Hkv, Hq // Hkv, b - a, D) / z
            out[at + a:at + b] = o.permute(2, 0, 1, 3).reshape(b - a, Hq, D).to(out.dtype)
            lse[at + a:at + b] = (m + torch.log(z))[..., 0].permute(2, 0, 1).reshape(b - a, Hq)
        at += n
    return out, lse


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
    req, bs = _requests(case), case["bs"]
    T = sum(n for _, n in req)
    fresh = sum(_blocks(c + n, bs) - _blocks(c, bs) for c, n in req)
    if case["op"] == "tables":
        # lengths, last held block and free blocks in; table entries, starts, lengths, slots and positions out
        return {"bytes": 8 * len(req) + 4 * sum(c % bs > 0 for c, _ in req) + 8 * fresh + 8 * len(req) + 4 + 12 * T + 8, "flops": 4 * T}
    if case["op"] == "append":
        return {"bytes": 2 * 2 * 2 * T * case["Hkv"] * case["D"] + 8 * T, "flops": 0}
    pairs, keys = _seen(case)
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    return {"bytes": 2 * 2 * T * Hq * D + 4 * T * Hq + 2 * 2 * keys * Hkv * D + 4 * sum(_blocks(c + n, bs) for c, n in req) + 8 * len(req),
            "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    h = _host(case, seed)
    table, taken, request, position, slot = _stepped(case, h)
    if case["op"] == "tables":
        return {"table": table, "query_start": np.concatenate([[0], np.cumsum(h["new"])]).astype(np.int32),
                "kv_len": h["cached"] + h["new"], "slot": slot, "position": position, "counts": np.array([taken, 0], np.int32)}
    if case["op"] == "append":
        return None   # nothing is computed
    if 4 * case["D"] * case["Hq"] * _seen(case)[0] > 4e12:
        return None
    st = prepare(case, seed)
    bs, D, Hkv = case["bs"], case["D"], case["Hkv"]
    G = case["Hq"] // Hkv
    window, causal = case.get("window", 0), case.get("causal", True)
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    begin = np.concatenate([[0], np.cumsum(h["new"])])
    for r in range(len(h["new"])):
        total, n = int(h["cached"][r] + h["new"][r]), int(h["new"][r])
        where = torch.from_numpy(table[r][np.arange(total) // bs].astype(np.int64) * bs + np.arange(total) % bs).cuda()
        for g in range(Hkv):
            K = st["k_cache"][where // bs, where % bs, g].double()
            V = st["v_cache"][where // bs, where % bs, g].double()
            step = max(1, _ROWS // (2 * total * G))
            for a in range(int(begin[r]), int(begin[r + 1]), step):
                b = min(a + step, int(begin[r + 1]))
                p = torch.from_numpy(position[a:b].astype(np.int64)).cuda()
                j = torch.arange(total, device="cuda")
                hidden = torch.zeros((b - a, total), dtype=torch.bool, device="cuda")
                if causal:
                    hidden |= j[None, :] > p[:, None]
                if window:
                    hidden |= j[None, :] <= p[:, None] - window
                s = torch.einsum("tgd,kd->tgk", st["q"][a:b, g * G:(g + 1) * G].double(), K) * st["scale"]
                s = s.masked_fill(hidden[:, None, :], -math.inf)
                z = torch.logsumexp(s, -1)
                out[a:b, g * G:(g + 1) * G] = torch.einsum("tgk,kd->tgd", torch.exp(s - z[..., None]), V)
                lse[a:b, g * G:(g + 1) * G] = z
    return out, lse
