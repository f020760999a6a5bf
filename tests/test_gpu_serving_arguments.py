"""Arguments of a serving step's calls at the ends of their ranges."""
import pytest

from test_gpu_serving import Batch, _i32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot
    return scoot


def test_the_largest_scale(S):
    """Scores of zero stay zero under the largest scale that is taken, and a larger one is refused: in the base-2 units of
    the softmax it is no longer finite, and a score of zero would be NaN."""
    b = Batch([(300, 40), (500, 1)], seed=1)
    b.q[:] = 0
    b.scale = 2.3e38
    with S.Context(torch.cuda.current_device()) as ctx:
        b.check(S, ctx)
        for scale in (2.4e38, 3.0e38):
            with pytest.raises(S.ScootError) as e:
                S.scoot_paged_attention(ctx, b.q, b.k, b.v, _i32(b.table), _i32(b.query_start), _i32(b.kv_len),
                                        torch.empty_like(b.q), scale)
            assert e.value.status == -1
        ctx.check()
