"""AttentionProbe's times are the GPU's: a slow host leaves them as they are."""
import time

import numpy as np
import pytest

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


@pytest.mark.parametrize("seqs", [4, 64])
def test_the_hosts_time_is_not_measured(ctx, monkeypatch, seqs):
    """Small steps, of some tens of microseconds on the GPU, whose queueing takes 3 ms each."""
    from paper_2408_04323_gb300 import serving
    n = 2 * seqs
    probe = serving.AttentionProbe(ctx, [20] * n, [5] * n, n_layers=1, n_heads=8, n_kv_heads=2, head_dim=64, cache_bytes=1 << 22)
    append = serving.S.scoot_kv_append

    def slow(*args, **kw):
        time.sleep(3e-3)
        append(*args, **kw)

    usual = probe.evaluate(seqs, 2048, 16, True)
    monkeypatch.setattr(serving.S, "scoot_kv_append", slow)
    late = probe.evaluate(seqs, 2048, 16, True)
    assert late["steps"] == usual["steps"]
    for got in (usual, late):
        assert 0 < got["tpot"] < 1e-3 and 0 < got["ttft"] < 1e-3 * got["steps"]


def test_a_step_queued_twice_is_the_same_step(ctx):
    from paper_2408_04323_gb300.serving import AttentionEngine
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((2, 96, 6, 64), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((2, 96, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    engines = [AttentionEngine(ctx, 2, 6, 2, 64, 16, 40, 4, 96, 200) for _ in range(2)]
    for new in ([30, 0, 17, 1], [1, 40, 1, 0], [0, 0, 0, 0], [16, 1, 1, 3]):
        outs = [torch.zeros_like(q) for _ in engines]
        for eng, out, times in zip(engines, outs, (1, 3)):
            eng.step(new, q, k, v, out, run=lambda launch: [launch() for _ in range(times)])
        ctx.check()
        a, b = engines
        assert torch.equal(*outs) and torch.equal(a.table, b.table) and torch.equal(a.kv_len, b.kv_len)
        assert np.array_equal(a.cached, b.cached) and a.free == b.free and a.blocks == b.blocks
