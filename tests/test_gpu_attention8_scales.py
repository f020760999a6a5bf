"""Attention over an 8-bit paged cache (scoot_paged_attention8) where scales lie far apart: blocks that a token does not see never
change its result, keys keep their codes beside others of any size, and scales reach the end of fp32."""
import numpy as np
import pytest

import serving8_ref as R8
from test_gpu_attention8 import F8, Batch, S, ctx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# (requests, heads, heads of keys, window, (request, key) in the block that some rows see and others do not): those of many rows
# for one kernel, of few for the other
UNSEEN = [([(440, 300), (90, 1)], 4, 2, 0, (0, 439)),        # a chunk's last block
          ([(500, 300)], 4, 1, 100, (0, 270)),               # in a window: a block that leaves and one that enters it
          ([(700, 600)], 2, 2, 40, (0, 115)),
          ([(98, 4), (33, 1)], 4, 2, 0, (0, 97)),            # few rows
          ([(996, 8)], 1, 1, 0, (0, 995)),
          ([(300, 8), (200, 3)], 4, 4, 10, (0, 279))]


def _seen(b, r, block, window):
    """Which tokens of request r see a key of its block's: bool [tokens]."""
    q0, q1, kv = int(b.query_start[r]), int(b.query_start[r + 1]), int(b.kv_len[r])
    p = kv - (q1 - q0) + np.arange(q1 - q0)
    first, last = block * b.bs, min(kv, (block + 1) * b.bs) - 1
    return (p >= first) & ((p - window < last) if window else True)


def _compare(b, out, lse, want, rows):
    o, z, eo, ez = want
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(got[rows]).all() and np.isfinite(gl[rows]).all()
    assert (np.abs(got - o)[rows] <= eo[rows]).all(), np.max((np.abs(got - o) / np.maximum(eo, 1e-30))[rows])
    assert (np.abs(gl - z)[rows] <= ez[rows]).all()


def _calls(b, S, ctx, **kw):
    """The call without and with the most that a request brings."""
    for most in (0, int(np.diff(b.query_start).max())):
        out, lse = b.run(S, ctx, max_new=most, **kw)
        ctx.check()
        yield out, lse


def _unseen(S, ctx, case, dtype, D, which, far, zeros=0):
    requests, H, Hkv, window, (r, key) = case
    b = Batch(requests, dtype=dtype, H=H, Hkv=Hkv, D=D, seed=D + len(requests), spread=1)
    b.scale[1][b.table[r, :zeros]] = 0.0
    want = b.want(window=window)   # as the tokens that do not see the block have it, whatever its scale
    block = key // b.bs
    for j in which:
        b.scale[j][int(b.table[r, block])] *= far
    rows = np.ones(len(b.q), bool)
    rows[int(b.query_start[r]):int(b.query_start[r + 1])] = ~_seen(b, r, block, window)
    assert rows.any() and not rows.all()
    for out, lse in _calls(b, S, ctx, window=window):
        _compare(b, out, lse, want, rows)


@pytest.mark.parametrize("case", UNSEEN)
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("far", [2.0 ** 26, 2.0 ** 40, 1.3 * 2.0 ** 60])
def test_keys_that_a_token_does_not_see_leave_no_trace(S, ctx, case, dtype, D, far):
    _unseen(S, ctx, case, dtype, D, (0,), far)


@pytest.mark.parametrize("case", UNSEEN)
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("far", [2.0 ** 3, 2.0 ** 5, 2.0 ** 12, 2.0 ** 23, 2.0 ** 40, 1.3 * 2.0 ** 60, 2.0 ** 110])
def test_values_that_a_token_does_not_see_leave_no_trace(S, ctx, case, dtype, D, far):
    _unseen(S, ctx, case, dtype, D, (1,), far)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("case,zeros", [(UNSEEN[2], 7), (UNSEEN[4], 60), (([(300, 8)], 4, 4, 10, (0, 279)), 17)])
def test_values_of_zero_beside_hidden_ones(S, ctx, case, dtype, D, zeros):
    """Tokens that see zeros alone, or these before others, where a block that they do not see is large."""
    _unseen(S, ctx, case, dtype, D, (1,), 2.0 ** 40, zeros)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("far", [2.0 ** 24, 2.0 ** 34, 2.0 ** 60])
@pytest.mark.parametrize("requests,H,Hkv", [([(400, 200)], 4, 2), ([(300, 2), (90, 1)], 4, 2)])
def test_keys_beside_much_larger_ones_keep_their_codes(S, ctx, D, far, requests, H, Hkv):
    """A block whose keys every token sees and gives no weight: its scores are far below the others', and further with a scale `far`
    times as large, which changes nothing but their distance."""
    b = Batch(requests, H=H, Hkv=Hkv, D=D, seed=5, spread=1)
    b.q = b.q.abs() + 0.5
    for r in range(len(requests)):
        c = b.cache[0].view(torch.uint8)[int(b.table[r, 3])]
        c[:] = torch.full_like(c, -64.0, dtype=torch.float32).to(F8).view(torch.uint8)
    at = [int(b.table[r, 3]) for r in range(len(requests))]
    # scores of -64 scale sum(q) / sqrt(D): 100 or more in size, that is a weight below e^-60 beside scores within some tens
    b.scale[0][at] = 0.25
    want = b.want()
    assert (want[1] > -25).all()
    b.scale[0][at] = 0.25 * far
    for out, lse in _calls(b, S, ctx):
        _compare(b, out, lse, want, slice(None))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [1.5 * 2.0 ** 126, 2.0 ** 127, 2.0 ** 126])
@pytest.mark.parametrize("requests", [[(200, 130)], [(300, 2), (90, 1)], [(150, 100), (33, 1)]])
@pytest.mark.parametrize("even", [True, False])
def test_values_scales_near_the_end_of_fp32(S, ctx, D, scale, requests, even):
    """With codes of 2^-9 to 2^-7, so that sums of values stay within fp32."""
    b = Batch(requests, dtype="bf16", H=4, Hkv=2, D=D, seed=9)
    c = b.cache[1].view(torch.uint8)
    c[:] = torch.where(c & 0x7F == 0x7F, c, c & 0x83)   # (the least codes, and the reserved ones where no request is)
    s = torch.isnan(b.scale[1])
    b.scale[1] = torch.where(s, b.scale[1], scale)
    if not even:
        b.scale[1][::2] *= 0.7
    b.check(S, ctx)
