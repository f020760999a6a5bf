"""AttentionEngine's record on the host, with a device that only remembers the calls (no GPU): what it refuses leaves it as it was."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")


class Event:
    def __init__(self, enable_timing=False):
        pass

    def record(self, stream=None):
        pass

    def synchronize(self):
        pass


@pytest.fixture()
def serving(monkeypatch):
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import serving
    calls = []
    for name in ("scoot_kv_tables", "scoot_kv_append", "scoot_paged_attention"):
        monkeypatch.setattr(serving.S, name, lambda *a, _n=name, **kw: calls.append(_n))
    monkeypatch.setattr(torch.cuda, "Event", Event)
    for name in ("empty", "zeros", "full"):   # on the host whatever device is asked for
        monkeypatch.setattr(torch, name, lambda *a, _f=getattr(torch, name), **kw: _f(*a, dtype=kw.get("dtype")))
    serving.calls = calls
    return serving


class Ctx:
    device = 0


def _engine(serving, seqs=4):
    return serving.AttentionEngine(Ctx(), 2, 4, 2, 64, 8, 20, seqs, 32, 64)


def _arrays(tokens=32, layers=2):
    q, k = torch.zeros((layers, tokens, 4, 64), dtype=torch.bfloat16), torch.zeros((layers, tokens, 2, 64), dtype=torch.bfloat16)
    return q, k, k.clone(), torch.zeros_like(q)


def _state(eng):
    return eng.cached.tolist(), list(eng.free), [list(b) for b in eng.blocks], [s is eng.stage[0] for s in eng.stage]


def test_a_step_and_the_rows_blocks(serving):
    eng = _engine(serving)
    assert eng.step([3, 0, 9, 0], *_arrays()) == 12
    assert eng.cached.tolist() == [3, 0, 9, 0] and eng.blocks == [[0], [], [1, 2], []]
    assert eng.step([6, 1, 0, 0], *_arrays()) == 7
    assert eng.cached.tolist() == [9, 1, 9, 0] and eng.blocks == [[0, 3], [4], [1, 2], []]
    eng.finish(2)
    assert eng.free == list(range(5, 20)) + [1, 2] and eng.cached.tolist() == [9, 1, 0, 0]
    assert serving.calls == (["scoot_kv_tables"] + ["scoot_kv_append", "scoot_paged_attention"] * 2) * 2


@pytest.mark.parametrize("new", [[1], [1, 1, 1], [1] * 5, 1, [[1, 1, 1, 1]], [5, -1, 0, 0], [-1, -1, -1, -1], [2 ** 31, 0, 0, 0],
                                 [2 ** 32 + 1, 0, 0, 0], [33, 0, 0, 0], []])
def test_counts_that_cannot_be_are_refused(serving, new):
    eng = _engine(serving)
    eng.step([3, 8, 1, 0], *_arrays())
    before, n = _state(eng), len(serving.calls)
    with pytest.raises(ValueError):
        eng.step(new, *_arrays())
    assert _state(eng) == before and len(serving.calls) == n


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("change", ["tokens", "layers", "heads", "dims"])
def test_arrays_that_do_not_fit_are_refused(serving, which, change):
    eng = _engine(serving)
    x = list(_arrays())
    x[which] = {"tokens": x[which][:, :5], "layers": x[which][:1], "heads": torch.cat([x[which]] * 2, 2)[:, :, :3],
                "dims": x[which][0]}[change]
    before = _state(eng)
    with pytest.raises(ValueError):
        eng.step([3, 3, 0, 0], *x)
    assert _state(eng) == before and not serving.calls


@pytest.mark.parametrize("prompts,outputs", [([5, 7], [1, 0]), ([0, 7], [1, 1]), ([5, -7], [1, 1]), ([5, 7], [1]), ([5], [1, 1]), ([], [])])
def test_requests_that_cannot_be_served_are_refused(serving, prompts, outputs):
    """An output of no token has no step at which it ends."""
    with pytest.raises(ValueError):
        serving.AttentionProbe(Ctx(), prompts, outputs)


@pytest.mark.parametrize("seqs,tokens", [(0, 64), (8, 0), (-1, 64)])
def test_a_configuration_without_sequences_or_tokens_serves_nothing(serving, seqs, tokens):
    assert serving.AttentionProbe(Ctx(), [5, 7], [2, 1]).evaluate(seqs, tokens, 16, True) is None
