"""Block tables with ids that cannot be, the least number of 32 bits among them: flagged, and the block counts as zeros, in
attention over 16-bit and 8-bit caches, for requests of few and of many rows."""
import numpy as np
import pytest

from test_gpu_attention8 import F8, Batch, S, ctx, _i32  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LEAST = -2 ** 31


@pytest.mark.parametrize("bad", [LEAST, LEAST + 1, -1, 2 ** 31 - 1])
@pytest.mark.parametrize("requests", [[(100, 1), (90, 1)], [(400, 300)], [(77, 2)]])
@pytest.mark.parametrize("eight", [True, False])
def test_an_id_that_a_row_sees_is_flagged(S, ctx, bad, requests, eight):
    b = Batch(requests, D=64, H=4, Hkv=2, seed=2)
    good = b.table[0, 4]
    if not eight:
        kv = [torch.nan_to_num(c.view(torch.uint8).view(F8).float() * s[:, None, :, None]).to(b.q.dtype) for c, s in zip(b.cache, b.scale)]

    def call():
        out = torch.full_like(b.q, 3.0)
        args = _i32(b.table), _i32(b.query_start), _i32(b.kv_len), out, b.factor
        if eight:
            S.scoot_paged_attention8(ctx, b.q, *b.cache, *b.scale, *args)
        else:
            S.scoot_paged_attention(ctx, b.q, *kv, *args)
        return out
    b.table[0, 4] = bad
    out = call()
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -4
    # as a block of zeros
    b.table[0, 4] = good
    if eight:
        for c, s in zip(b.cache, b.scale):
            c.view(torch.uint8)[int(good)] = 0
            s[int(good)] = 0.0
    else:
        for c in kv:
            c[int(good)] = 0
    want = call()
    ctx.check()
    assert torch.equal(out, want)


@pytest.mark.parametrize("bad", [LEAST, -1])
def test_an_id_that_no_row_sees_is_not(S, ctx, bad):
    b = Batch([(400, 300), (200, 1)], D=64, H=4, Hkv=2, seed=2)
    want = b.run(S, ctx, window=60)
    b.table[0, :2] = bad
    b.table[1, :8] = bad
    got = b.run(S, ctx, window=60)
    ctx.check()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
