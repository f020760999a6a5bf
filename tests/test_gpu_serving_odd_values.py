"""Values that are infinite or NaN, seen by some tokens: they reach those, in their dimension, as the definition has it (every
probability is positive), wherever the key lies in its tile, however the rows are laid out, and however small the weight."""
import numpy as np
import pytest

import serving_ref as R
from test_gpu_serving import Batch

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot
    return scoot


def _check(S, b, **kw):
    with S.Context(torch.cuda.current_device()) as ctx:
        out, lse = b.run(S, ctx, **kw)
        ctx.check()
    o, z, eo, ez = b.want(**kw)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    odd = ~np.isfinite(o)
    assert odd.any()
    assert np.array_equal(got[odd], o[odd], equal_nan=True)
    assert (np.abs(got[~odd] - o[~odd]) <= eo[~odd]).all()
    assert (np.abs(gl - z) <= ez).all()


# 2, 16, 40 and 96 rows of a token: four copies, four, two and one
@pytest.mark.parametrize("H,Hkv", [(4, 2), (16, 1), (40, 1), (96, 1)])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_single_tokens(S, H, Hkv, D, dtype, bad):
    """A key inside the sequence for each quarter of a tile, and one in a later tile, each in a dimension of its own."""
    b = Batch([(700, 1), (300, 1)], dtype=dtype, H=H, Hkv=Hkv, D=D, seed=H)
    for i, key in enumerate((128 + 5, 128 + 40, 128 + 70, 128 + 127, 0, 600)):
        b.v[b.at(0, key)][..., Hkv - 1, 9 * i + 3] = bad
    _check(S, b)
    _check(S, b, window=400)


@pytest.mark.parametrize("first,second", [(INF, INF), (INF, -INF), (-INF, -INF), (NAN, INF)])
@pytest.mark.parametrize("keys", [(130, 135), (130, 170), (130, 300), (130, 699)])
def test_two_values_of_a_dimension(S, first, second, keys):
    b = Batch([(700, 1)], H=8, Hkv=2, D=64, seed=2)
    for bad, key in zip((first, second), keys):
        b.v[b.at(0, key)][..., 0, 33] = bad
    _check(S, b)


@pytest.mark.parametrize("requests,H,Hkv", [([(700, 1)], 8, 2), ([(500, 2), (90, 1)], 40, 1), ([(400, 300)], 4, 2), ([(640, 200)], 8, 1),
                                            ([(20000, 1)], 8, 1), ([(9000, 1)], 96, 1), ([(9000, 40)], 4, 1)])
@pytest.mark.parametrize("D,dtype", [(64, "fp16"), (128, "bf16")])
def test_weights_that_round_to_zero(S, requests, H, Hkv, D, dtype):
    """Scores of a spread of hundreds: most weights are zero in the cache's type, many in fp32."""
    b = Batch(requests, dtype=dtype, H=H, Hkv=Hkv, D=D, seed=D)
    b.scale = 4.0
    kv, n = requests[0]
    rng = np.random.default_rng(kv)
    for i, key in enumerate(rng.choice(kv - n, 12, replace=False)):
        b.v[b.at(0, int(key))][..., 0, 5 * i] = (INF, -INF, NAN)[i % 3]
    if n > 1:
        b.v[b.at(0, kv - n // 2)][..., 0, 62] = -INF  # that some of the new tokens see
    _check(S, b)


def test_every_value(S):
    """A cache of infinities, and one of NaN."""
    for bad in (INF, NAN):
        b = Batch([(260, 1), (300, 130)], H=8, Hkv=2, D=64, seed=8)
        b.v[:] = bad
        _check(S, b)
