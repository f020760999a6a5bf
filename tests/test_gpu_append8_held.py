"""Appends to an 8-bit cache (scoot_kv_append8) whose blocks hold a scale that cannot be: the earlier tokens become zeros whatever
their codes."""
import numpy as np
import pytest

import serving8_ref as R8
from test_gpu_rotary import DTYPE, F8, S, _codes, _dev, _np, _randn, ctx  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held", [float("nan"), float("inf"), -float("inf"), -1.0])
@pytest.mark.parametrize("D,dtype", [(64, "fp16"), (128, "bf16")])
def test_codes_under_a_scale_that_cannot_be_become_zeros(S, ctx, held, D, dtype):
    """The codes that the format reserves for NaN among them, as in memory that nobody has written."""
    x = _randn((2, 2, D), dtype, 2)
    old = torch.randint(0, 256, (1, 8, 2, D), generator=torch.Generator().manual_seed(3), dtype=torch.uint8).cuda()
    old[:, :, :, ::5] = 0x7F
    old[:, :, :, 1::5] = 0xFF
    kc, vc = old.clone().view(F8), old.clone().view(F8)
    ks, vs = (torch.full((1, 2), held, device="cuda") for _ in range(2))
    S.scoot_kv_append8(ctx, x, x, _dev([3, 4], np.int64), kc, vc, ks, vs)
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -1
    need = R8.least_scale(np.abs(_np(x)).max((0, 2)))
    for c, s in ((kc, ks), (vc, vs)):
        assert np.array_equal(_np(s)[0], need)
        got = _codes(c)[0]
        assert (got[:3] == 0).all()
        assert np.array_equal(got[3:5], R8.code_of(_np(x) / need[None, :, None]))
        assert torch.equal(c.view(torch.uint8)[0, 5:], old[0, 5:])
