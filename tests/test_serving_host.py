"""A serving step's entry points on the host: a missing context is an error code, and the plain forms that the GPU tests
compare with hold on cases worked by hand."""
import numpy as np
import pytest

import serving_ref as R


@pytest.fixture(scope="module")
def L():
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot
    return scoot.lib()


def test_a_missing_context_is_an_error_code(L):
    assert L.scoot_kv_tables(None, None, None, 0, 16, 1, None, 0, None, 0, None, None, None, None, 0, None, None) == -1
    assert L.scoot_kv_append(None, None, None, 0, 0, None, 0, 0, None, 0, None, None, None) == -1
    assert L.scoot_paged_attention(None, None, None, 0, 0, 1, 0, None, None, 0, None, 0, None, None, 1.0, 1, 0, None, 0, 0,
                                   None, None) == -1


def test_tables_by_hand():
    """Blocks of 8: request 0 holds one block with 6 tokens and brings 3 (one more block), request 1 starts with 9 tokens
    (two blocks), request 2 wants two but one is left, request 3 fits in its own block."""
    table = np.array([[4, -1, -1], [-1, -1, -1], [-1, -1, -1], [7, -1, -1]])
    t, start, kv, slot, pos, counts = R.tables(np.array([6, 0, 0, 2]), np.array([3, 9, 16, 1]), table, 8, 10, [5, 0, 3, 9], 30)
    assert t.tolist() == [[4, 5, -1], [0, 3, -1], [-1, -1, -1], [7, -1, -1]]
    assert start.tolist() == [0, 3, 12, 28, 29] and kv.tolist() == [9, 9, 0, 3] and counts.tolist() == [3, 1]
    assert slot[:3].tolist() == [38, 39, 40] and slot[3:12].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, 24]
    assert (slot[12:28] == -1).all() and slot[28] == 58 and slot[29] == -1
    assert pos[:3].tolist() == [6, 7, 8] and pos[28] == 2 and pos[29] == 0


def test_attention_by_hand():
    """One dimension apart from zeros: scores 0 and ln 3 give weights 1/4 and 3/4; a window of one leaves the last key; a
    token before the sequence's start sees nothing."""
    q = np.zeros((3, 1, 64))
    q[:, 0, 0] = 1.0
    k = np.zeros((2, 8, 1, 64))
    v = np.zeros((2, 8, 1, 64))
    k[1, 1, 0, 0] = np.log(3.0)
    v[1, 0, 0, 2], v[1, 1, 0, 2] = 4.0, 8.0
    args = (q, k, v, np.array([[1]]), [0, 3], [2], 1.0)
    out, lse, e_out, e_lse = R.attention(*args)
    assert np.allclose(out[:, 0, 2], [0.0, 4.0, 7.0]) and np.isneginf(lse[0, 0]) and np.allclose(lse[1:, 0], [0.0, np.log(4.0)])
    assert (e_out[2, 0, 2] > 0) and (e_out[2, 0, 2] < 0.1)
    assert np.allclose(R.attention(*args, window=1)[0][:, 0, 2], [0.0, 4.0, 8.0])
    assert np.allclose(R.attention(*args, causal=False)[0][:, 0, 2], [7.0, 7.0, 7.0])
