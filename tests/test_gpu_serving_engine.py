"""The attention part of an engine's steps (serving.AttentionEngine) against plain 64-bit attention over what each sequence
was given, and the probe that evaluates configurations with it."""
import numpy as np
import pytest

import serving_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot as S
    with S.Context(torch.cuda.current_device()) as c:
        yield c


@pytest.mark.parametrize("dtype,block,window", [("bf16", 16, 0), ("fp16", 8, 20)])
def test_steps_attend_to_what_each_sequence_was_given(ctx, dtype, block, window):
    from paper_2408_04323_gb300.serving import AttentionEngine
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    L, H, Hkv, D, seqs = 2, 6, 2, 64, 4
    eng = AttentionEngine(ctx, L, H, Hkv, D, block, 40, seqs, 96, 200, dt, window)
    rng = np.random.default_rng(3)
    K = [[np.zeros((0, Hkv, D)) for _ in range(seqs)] for _ in range(L)]
    V = [[np.zeros((0, Hkv, D)) for _ in range(seqs)] for _ in range(L)]
    plan = [[30, 0, 17, 1], [1, 40, 1, 0], [1, 1, 33, 9], "finish 2", [1, 1, 50, 1], [0, 0, 0, 0], [16, 1, 1, 3], "finish 0", [64, 1, 1, 1]]
    for new in plan:
        if isinstance(new, str):
            r = int(new.split()[1])
            eng.finish(r)
            for layer in range(L):
                K[layer][r], V[layer][r] = np.zeros((0, Hkv, D)), np.zeros((0, Hkv, D))
            continue
        n = sum(new)
        q = torch.randn((L, 96, H, D), device="cuda").to(dt)
        k, v = (torch.randn((L, 96, Hkv, D), device="cuda").to(dt) for _ in range(2))
        out = torch.empty_like(q)
        assert eng.step(new, q, k, v, out) == n
        ctx.check()
        start = np.concatenate([[0], np.cumsum(new)])
        for layer in range(L):
            for r in range(seqs):
                K[layer][r] = np.concatenate([K[layer][r], k[layer, start[r]:start[r + 1]].double().cpu().numpy()])
                V[layer][r] = np.concatenate([V[layer][r], v[layer, start[r]:start[r + 1]].double().cpu().numpy()])
            lens = np.array([len(x) for x in K[layer]])
            assert (lens == eng.cached).all()
            kc, vc = (np.zeros((seqs, max(1, lens.max()), Hkv, D)) for _ in range(2))  # a block per sequence
            for r in range(seqs):
                kc[r, :lens[r]], vc[r, :lens[r]] = K[layer][r], V[layer][r]
            o, _, eo, _ = R.attention(q[layer, :n].double().cpu().numpy(), kc, vc, np.arange(seqs)[:, None], start, lens, D ** -0.5,
                                      window=window, unit=R.UNIT[dtype])
            assert (np.abs(out[layer, :n].double().cpu().numpy() - o) <= eo).all()
    held = sorted(b for row in eng.blocks for b in row)
    assert sorted(held + eng.free) == list(range(40))
    for r in range(seqs):  # the host's record of the blocks is the device's
        assert eng.table[r, :len(eng.blocks[r])].tolist() == eng.blocks[r]


def test_a_step_that_cannot_be_is_refused_before_it_starts(ctx):
    from paper_2408_04323_gb300.serving import AttentionEngine
    eng = AttentionEngine(ctx, 1, 2, 1, 64, 16, 3, 2, 40, 64)
    q = torch.zeros((1, 40, 2, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((1, 40, 1, 64), dtype=torch.bfloat16, device="cuda")
    for bad, error in (([41, 0], ValueError), ([0, 65], ValueError), ([20, 20], RuntimeError)):
        with pytest.raises(error):
            eng.step(bad, q, k, k, q.clone())
    assert (eng.cached == 0).all() and len(eng.free) == 3


@pytest.mark.parametrize("chunked", [False, True])
def test_probe_serves_every_request(ctx, chunked):
    from paper_2408_04323_gb300.serving import AttentionProbe
    rng = np.random.default_rng(1)
    prompts, outputs = rng.integers(5, 300, 12), rng.integers(1, 9, 12)
    probe = AttentionProbe(ctx, prompts, outputs, n_layers=1, n_heads=8, n_kv_heads=2, head_dim=64, cache_bytes=1 << 21)
    got = probe.evaluate(8, 512, 16, chunked)
    assert got is not None and got["ttft"] > 0 and got["tpot"] > 0 and got["throughput"] > 0
    # at least as many steps as the longest output and as the tokens over the budget
    assert got["steps"] >= max(int(outputs.max()), -(-int(prompts.sum()) // 512))
    assert probe.evaluate(8, 100, 16, False) is None       # a prompt longer than a step's tokens, not chunked
    small = AttentionProbe(ctx, prompts, outputs, n_layers=1, n_heads=8, n_kv_heads=2, head_dim=64, cache_bytes=1 << 14)
    assert small.evaluate(8, 512, 16, True) is None         # a request longer than the cache


def test_the_loop_tunes_on_the_probe(ctx):
    from paper_2408_04323_gb300.serving import AttentionProbe, tune
    rng = np.random.default_rng(2)
    probe = AttentionProbe(ctx, rng.integers(20, 200, 8), rng.integers(2, 6, 8), n_layers=1, n_heads=4, n_kv_heads=1, head_dim=64,
                           cache_bytes=1 << 22)
    seen = tune(ctx, probe, rounds=1, n_init=5, q=2, say=lambda *a: None)
    assert len(seen) == 7
    for cfg, got in seen:
        assert cfg["max_num_batched_tokens"] >= cfg["max_num_seqs"]
        assert got is None or got["throughput"] > 0
