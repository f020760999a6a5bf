"""The attention part of an engine's steps, and an evaluation of engine configurations on it.

Algorithm 1 evaluates a suggested configuration by a stress test of the engine.  Of the parameters that it tunes (Section 2,
Table 1), the most sequences and most batched tokens of a step, the block size, chunked prefill and the memory
utilisation act on one part of the engine's step: which tokens it takes, where their keys and values go, and the
attention over them.  `AttentionEngine` runs that part, `AttentionProbe` serves a list of requests with it under a
configuration and reports the latencies and the throughput, which `loop.TuningLoop` takes as objectives:

    python -m paper_2408_04323_gb300.serving

The step's work is the library's: scoot_kv_tables once, then scoot_kv_append and scoot_paged_attention per layer, or
with rotary positions scoot_kv_append_rotary, or over a cache of 8-bit floats scoot_kv_append8 and
scoot_paged_attention8.
"""
from __future__ import annotations

import numpy as np
import torch

from . import scoot as S


class AttentionEngine:
    """Up to max_seqs sequences over one paged cache per layer.

    A sequence has a row (0 .. max_seqs - 1) for as long as it runs; a step gives every row a number of new tokens (0 for
    rows that sit out).  Lengths and tables live on the device; the host keeps the lengths and each row's blocks as
    well, by the rule that the device follows (blocks from the front of the free list, in the rows' order), and so knows
    what is free without asking.  Everything is asynchronous on the current stream.

    rotation (a scoot.Rotation): keys are turned by their tokens' positions as they go into the cache, and queries, in a copy
    of the engine's, before they meet them.  cache8: the caches hold e4m3 codes with a scale per block and head, half the
    bytes; dtype is that of queries, keys, values and outputs either way.  Single tokens over much cached are faster with it, by up
    to 1.8 times; long prompts are slower, by up to 1.4 times, and so are appends, and a lone short sequence (by a tenth)."""

    def __init__(self, ctx: S.Context, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, block_size: int,
                 n_blocks: int, max_seqs: int, max_tokens: int, max_len: int, dtype=torch.bfloat16, window: int = 0,
                 rotation: S.Rotation | None = None, cache8: bool = False):
        if rotation is not None:
            S._rotation(rotation, ctx.device)
            if rotation.rot_dim > head_dim:
                raise ValueError(f"a rotation of {rotation.rot_dim} dimensions for heads of {head_dim}")
        self.ctx, self.block_size, self.n_blocks = ctx, int(block_size), int(n_blocks)
        self.max_tokens, self.max_len, self.window = int(max_tokens), int(max_len), int(window)
        self.scale = head_dim ** -0.5
        dev = torch.device("cuda", ctx.device)
        shape = (n_layers, n_blocks, block_size, n_kv_heads, head_dim)
        self.rotation, self.cache8 = rotation, bool(cache8)
        self.k_cache, self.v_cache = (torch.empty(shape, dtype=torch.float8_e4m3fn if cache8 else dtype, device=dev) for _ in range(2))
        if cache8:
            self.k_scale, self.v_scale = (torch.zeros((n_layers, n_blocks, n_kv_heads), dtype=torch.float32, device=dev) for _ in range(2))
        if rotation is not None:  # a layer's turned queries (not in place: a step's work may be queued more than once)
            self.turned = torch.empty((max_tokens, n_heads, head_dim), dtype=dtype, device=dev)
        width = -(-max_len // block_size)
        self.table = torch.full((max_seqs, width), -1, dtype=torch.int32, device=dev)
        # cached and new lengths, and the free blocks that the step takes: one copy from two pinned buffers in turn
        self.inputs = torch.zeros(2 * max_seqs + n_blocks, dtype=torch.int32, device=dev)
        self.stage = [(torch.zeros(2 * max_seqs + n_blocks, dtype=torch.int32, pin_memory=True), torch.cuda.Event()) for _ in range(2)]
        self.query_start = torch.zeros(max_seqs + 1, dtype=torch.int32, device=dev)
        self.kv_len = torch.zeros(max_seqs, dtype=torch.int32, device=dev)
        self.slot = torch.empty(max_tokens, dtype=torch.int64, device=dev)
        self.position = torch.empty(max_tokens, dtype=torch.int32, device=dev)
        self.counts = torch.zeros(2, dtype=torch.int32, device=dev)
        self.free = list(range(n_blocks))
        self.cached = np.zeros(max_seqs, np.int32)
        self.blocks: list[list[int]] = [[] for _ in range(max_seqs)]

    def blocks_for(self, row: int, n_new: int) -> int:
        """Blocks that n_new more tokens of the row would take."""
        return -(-(int(self.cached[row]) + n_new) // self.block_size) - len(self.blocks[row])

    def step(self, new, q, k, v, out, run=None):
        """new [max_seqs]: new tokens per row; q, out [layers][tokens][heads][dim] and k, v [layers][tokens][kv heads][dim]
        with the rows' tokens back to back.  Fills out; returns the number of tokens.  A step that cannot be (counts,
        lengths, blocks or shapes) is refused before anything is changed.  run: called in place of the function that it is
        given, which queues the step's work on the current stream; it may do so more than once, with the same result."""
        new = np.asarray(new, np.int64)
        if new.shape != self.cached.shape or new.min(initial=0) < 0:
            raise ValueError(f"new must be {len(self.cached)} counts, none of them negative, got {new.tolist()}")
        n = int(new.sum())
        if n > self.max_tokens or (self.cached + new).max(initial=0) > self.max_len:
            raise ValueError(f"{n} tokens, or a sequence of {(self.cached + new).max(initial=0)}, beyond {self.max_tokens} "
                             f"and {self.max_len}")
        layers, (kv_heads, dim) = len(self.k_cache), self.k_cache.shape[-2:]
        for name, x, heads in (("q", q, q.shape[-2]), ("k", k, kv_heads), ("v", v, kv_heads), ("out", out, q.shape[-2])):
            if x.dim() != 4 or len(x) < layers or x.shape[1] < n or x.shape[2:] != (heads, dim) or heads % kv_heads:
                raise ValueError(f"{name} must be [{layers}][at least {n}][{heads}][{dim}], the query heads a multiple of {kv_heads}, "
                                 f"got {tuple(x.shape)}")
        if self.rotation is not None and q.shape[-2] != self.turned.shape[1]:
            raise ValueError(f"q has {q.shape[-2]} heads, and the engine was made for {self.turned.shape[1]}")
        need = [self.blocks_for(r, int(c)) for r, c in enumerate(new)]
        if sum(need) > len(self.free):
            raise RuntimeError(f"{sum(need)} blocks wanted, {len(self.free)} free")
        rows, taken = len(new), sum(need)
        size = 2 * rows + taken
        stage, copied = self.stage[0]
        self.stage.reverse()
        copied.synchronize()  # of the step before last
        host = stage.numpy()
        host[:rows], host[rows:2 * rows], host[2 * rows:size] = self.cached, new, self.free[:taken]
        slot, position = self.slot[:n], self.position[:n]

        def launch():
            self.inputs[:size].copy_(stage[:size], non_blocking=True)
            copied.record()
            S.scoot_kv_tables(self.ctx, self.inputs[:rows], self.inputs[rows:2 * rows], self.table, self.block_size,
                              self.n_blocks, self.inputs[2 * rows:size], self.query_start, self.kv_len, slot, position, self.counts)
            for layer in range(len(self.k_cache)):
                self._layer(layer, q[layer, :n], k[layer, :n], v[layer, :n], slot, position, out[layer, :n], int(new.max(initial=0)))

        launch() if run is None else run(launch)
        for r, m in enumerate(need):
            self.blocks[r] += self.free[:m]
            del self.free[:m]
        self.cached += new.astype(np.int32)
        return n

    def _layer(self, layer, q, k, v, slot, position, out, max_new):
        ctx, kc, vc = self.ctx, self.k_cache[layer], self.v_cache[layer]
        turned = q if self.rotation is None else self.turned[:len(q)]
        if self.cache8:
            scales = self.k_scale[layer], self.v_scale[layer]
            if self.rotation is None:
                S.scoot_kv_append8(ctx, k, v, slot, kc, vc, *scales)
            else:
                S.scoot_kv_append8(ctx, k, v, slot, kc, vc, *scales, self.rotation, position, q, turned)
            S.scoot_paged_attention8(ctx, turned, kc, vc, *scales, self.table, self.query_start, self.kv_len, out, self.scale,
                                     window=self.window, max_new=max_new)
            return
        if self.rotation is None:
            S.scoot_kv_append(ctx, k, v, slot, kc, vc)
        else:
            S.scoot_kv_append_rotary(ctx, self.rotation, k, v, slot, position, kc, vc, q, turned)
        S.scoot_paged_attention(ctx, turned, kc, vc, self.table, self.query_start, self.kv_len, out, self.scale, window=self.window)

    def finish(self, row: int) -> None:
        """Gives the row's blocks back."""
        self.free += self.blocks[row]
        self.blocks[row] = []
        self.cached[row] = 0


class AttentionProbe:
    """Serves requests (prompt and output lengths, all there at the start) with an AttentionEngine under a configuration
    and measures the steps on the GPU: the time of its work alone, not that of the host, which plans and queues each step
    while a delay holds the GPU back.  Stands in for the engine in Algorithm 1's evaluation where only the
    attention's share of a step is wanted, or to try the loop without an engine: queries, keys and values are random.
    rotation and cache8 as in AttentionEngine: cache_bytes then hold about twice the blocks."""

    SHORTEST_DELAY, LONGEST_DELAY = 1 << 12, 1 << 22  # iterations of the delay's kernel: some 70 us and 70 ms

    def __init__(self, ctx: S.Context, prompts, outputs, n_layers: int = 2, n_heads: int = 32, n_kv_heads: int = 8,
                 head_dim: int = 128, cache_bytes: int = 1 << 30, dtype=torch.bfloat16, seed: int = 0,
                 rotation: S.Rotation | None = None, cache8: bool = False):
        self.ctx, self.prompts, self.outputs = ctx, [int(p) for p in prompts], [int(o) for o in outputs]
        if len(self.prompts) != len(self.outputs) or not self.prompts or min(self.prompts + self.outputs) < 1:
            raise ValueError("prompts and outputs must be one length each per request, all of them at least 1")
        self.shape = (n_layers, n_heads, n_kv_heads, head_dim)
        self.cache_bytes, self.dtype, self.seed = int(cache_bytes), dtype, seed
        self.rotation, self.cache8 = rotation, bool(cache8)
        self.delay = self.SHORTEST_DELAY  # about as long as queueing a step takes

    def _timed(self, marks, sink):
        """A step's run: queues it behind a delay, and again behind a longer one if the GPU came to the step before all
        of it was queued, so that its marks hold no time in which the GPU waits for the host."""
        def run(launch):
            while True:
                start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                S.scoot_probe_fma(self.ctx, False, 1, self.delay, sink)
                start.record()
                launch()
                stop.record()
                if not start.query() or self.delay >= self.LONGEST_DELAY:
                    marks.append((start, stop))
                    self.delay = max(self.SHORTEST_DELAY, self.delay - self.delay // 64)  # (a pause of the host passes)
                    return
                self.delay *= 2
        return run

    def evaluate(self, max_num_seqs: int, max_num_batched_tokens: int, block_size: int, chunked_prefill: bool,
                 memory_utilization: float = 0.9):
        """{"ttft", "tpot": mean seconds, "throughput": output tokens per second, "steps"}, or None if the configuration
        cannot serve the requests (a prompt that fits neither the step nor the cache: the engine would crash; or steps of no
        sequence or token)."""
        L, H, Hkv, D = self.shape
        longest = max(p + o for p, o in zip(self.prompts, self.outputs))
        per_block = 2 * L * Hkv * (block_size * D + 4 if self.cache8 else 2 * block_size * D)  # (4: a scale)
        n_blocks = int(self.cache_bytes * memory_utilization) // per_block
        if n_blocks < -(-longest // block_size) or (not chunked_prefill and max(self.prompts) > max_num_batched_tokens) or \
                min(max_num_seqs, max_num_batched_tokens) < 1:
            return None
        seqs, budget = min(max_num_seqs, len(self.prompts)), max_num_batched_tokens
        eng = AttentionEngine(self.ctx, L, H, Hkv, D, block_size, n_blocks, seqs, budget, longest, self.dtype, rotation=self.rotation,
                              cache8=self.cache8)
        gen = torch.Generator(device="cuda").manual_seed(self.seed)
        q = torch.randn((L, budget, H, D), generator=gen, device="cuda", dtype=torch.float32).to(self.dtype)
        k, v = (torch.randn((L, budget, Hkv, D), generator=gen, device="cuda", dtype=torch.float32).to(self.dtype) for _ in range(2))
        out = torch.empty_like(q)
        warm = AttentionEngine(self.ctx, 1, H, Hkv, D, block_size, 1, 1, 1, 1, self.dtype, rotation=self.rotation,
                               cache8=self.cache8)  # code and workspace are there
        warm.step([1], q[:1], k[:1], v[:1], out[:1])
        waiting = list(range(len(self.prompts)))[::-1]
        row_of: list[int | None] = [None] * seqs   # the request of each row
        left = np.zeros(seqs, int)                 # prompt tokens still to take
        promised = 0                               # blocks that running requests may still take
        marks, first, last = [], {}, {}
        timed = self._timed(marks, torch.zeros(1, device="cuda"))
        while waiting or any(r is not None for r in row_of):
            for row in range(seqs):                # admit while the cache has room for the whole request
                if row_of[row] is not None or not waiting:
                    continue
                need = -(-(self.prompts[waiting[-1]] + self.outputs[waiting[-1]]) // block_size)
                if need + promised > len(eng.free):
                    break
                row_of[row] = waiting.pop()
                left[row] = self.prompts[row_of[row]]
                promised += need
            new = np.zeros(seqs, np.int32)
            prefill = [r for r in range(seqs) if row_of[r] is not None and left[r] > 0]
            decode = [r for r in range(seqs) if row_of[r] is not None and left[r] == 0]
            room = budget
            if chunked_prefill or not prefill:     # decodes first, and what is left of the budget for prompts
                for r in decode[:room]:
                    new[r] = 1
                    room -= 1
            for r in prefill:
                n = min(int(left[r]), room)
                if n < left[r] and not chunked_prefill:
                    continue
                new[r] = n
                room -= n
            before = len(eng.free)
            eng.step(new, q, k, v, out, timed)
            promised -= before - len(eng.free)
            for r in np.flatnonzero(new):
                i = row_of[r]
                left[r] = max(0, left[r] - new[r])
                if left[r]:
                    continue
                first.setdefault(i, len(marks) - 1)
                if eng.cached[r] == self.prompts[i] + self.outputs[i] - 1:   # the last token needs no step
                    last[i] = len(marks) - 1
                    promised -= -(-(self.prompts[i] + self.outputs[i]) // block_size) - len(eng.blocks[r])
                    eng.finish(int(r))
                    row_of[r] = None
        torch.cuda.synchronize()
        self.ctx.check()
        at = np.cumsum([a.elapsed_time(b) * 1e-3 for a, b in marks])
        tpot = [(at[last[i]] - at[first[i]]) / (o - 1) for i, o in enumerate(self.outputs) if o > 1]
        return {"ttft": float(np.mean([at[first[i]] for i in first])), "tpot": float(np.mean(tpot)) if tpot else 0.0,
                "throughput": sum(self.outputs) / float(at[-1]), "steps": len(marks)}


BLOCK_SIZES = (8, 16, 32)


def tune(ctx: S.Context, probe: AttentionProbe, rounds: int = 4, n_init: int = 8, q: int = 2, seed: int = 0, say=print):
    """Algorithm 1 with the probe as its evaluation: minimise the time to the first token and the time per token over the
    most sequences, the most batched tokens, the block size, chunked prefill and the memory utilisation.  Returns the
    evaluated configurations as [(configuration, result)]."""
    from .loop import TuningLoop
    space = np.zeros(5, np.dtype([("kind", "<i4"), ("n_choices", "<i4"), ("lo", "<f4"), ("hi", "<f4")]))
    space[:] = [(S.INT_LOG, 0, 1, 256), (S.INT_LOG, 0, 64, 8192), (S.CATEGORICAL, 3, 0, 0), (S.CATEGORICAL, 2, 0, 0),
                (S.CONTINUOUS, 0, 0.5, 0.95)]
    clauses = np.zeros(1, np.dtype([("n_guard", "<i4"), ("guard_param", "<i4", (2,)), ("guard_value", "<i4", (2,)), ("n_term", "<i4"),
                                    ("term_param", "<i4", (4,)), ("coef", "<i8", (4,)), ("rhs", "<i8")]))
    clauses[0]["n_term"], clauses[0]["term_param"][:2], clauses[0]["coef"][:2] = 2, (1, 0), (1, -1)  # tokens >= sequences
    loop = TuningLoop(ctx, space, clauses, n_obj=2, q=q, pool=4096, seed=seed)
    seen = []

    def evaluate(words):
        y, ok = np.zeros((2, words.shape[1])), np.zeros(words.shape[1], bool)
        for j in range(words.shape[1]):
            w = words[:, j]
            cfg = {"max_num_seqs": int(w[0]), "max_num_batched_tokens": int(w[1]), "block_size": BLOCK_SIZES[int(w[2])],
                   "chunked_prefill": bool(w[3]), "memory_utilization": float(w[4:5].view(np.float32)[0])}
            got = probe.evaluate(**cfg)
            seen.append((cfg, got))
            say(cfg, got)
            if got is not None:
                ok[j], y[:, j] = True, (-got["ttft"], -got["tpot"])
        loop.observe(words, y, ok)

    evaluate(loop.initial_design(n_init))
    for _ in range(rounds):
        evaluate(loop.suggest())
    return seen


def main() -> None:
    rng = np.random.default_rng(0)
    prompts, outputs = rng.integers(32, 2048, 64), rng.integers(16, 128, 64)
    with S.Context(torch.cuda.current_device()) as ctx:
        seen = tune(ctx, AttentionProbe(ctx, prompts, outputs))
    best = min((s for s in seen if s[1] is not None), key=lambda s: s[1]["tpot"])
    print("least time per token:", *best)


if __name__ == "__main__":
    main()
