"""AttentionEngine with rotary positions and with an 8-bit cache on the host, with a device that only remembers the calls (no GPU)."""
import pytest

torch = pytest.importorskip("torch")

APPEND = {(False, False): "scoot_kv_append", (True, False): "scoot_kv_append_rotary", (False, True): "scoot_kv_append8",
          (True, True): "scoot_kv_append8"}


class Event:
    def __init__(self, enable_timing=False):
        pass

    def record(self, stream=None):
        pass

    def synchronize(self):
        pass


class Ctx:
    device = 0


@pytest.fixture()
def serving(monkeypatch):
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import serving
    calls = []
    for name in {"scoot_kv_tables", "scoot_paged_attention", "scoot_paged_attention8", *APPEND.values()}:
        monkeypatch.setattr(serving.S, name, lambda *a, _n=name, **kw: calls.append((_n, a, kw)))
    monkeypatch.setattr(torch.cuda, "Event", Event)
    for name in ("empty", "zeros", "full"):   # on the host whatever device is asked for
        monkeypatch.setattr(torch, name, lambda *a, _f=getattr(torch, name), **kw: _f(*a, dtype=kw.get("dtype")))
    serving.calls = calls
    return serving


def _rotation(serving, rot_dim=64, device=0):
    r = object.__new__(serving.S.Rotation)
    r.rot_dim, r.device, r.ref = rot_dim, device, None
    return r


def _engine(serving, turn, cache8, **kw):
    return serving.AttentionEngine(Ctx(), 2, 4, 2, 64, 8, 20, 4, 32, 64, rotation=_rotation(serving) if turn else None, cache8=cache8, **kw)


def _arrays(heads=4, tokens=32):
    q, k = torch.zeros((2, tokens, heads, 64), dtype=torch.bfloat16), torch.zeros((2, tokens, 2, 64), dtype=torch.bfloat16)
    return q, k, k.clone(), torch.zeros_like(q)


@pytest.mark.parametrize("turn", [False, True])
@pytest.mark.parametrize("cache8", [False, True])
def test_the_calls_of_a_step(serving, turn, cache8):
    eng, x = _engine(serving, turn, cache8), _arrays()
    assert eng.step([3, 0, 9, 0], *x) == 12
    names = [c[0] for c in serving.calls]
    assert names == ["scoot_kv_tables"] + [APPEND[turn, cache8], "scoot_paged_attention8" if cache8 else "scoot_paged_attention"] * 2
    for layer, (append, attend) in enumerate(zip(serving.calls[1::2], serving.calls[2::2])):
        caches = [t.data_ptr() for t in (eng.k_cache[layer], eng.v_cache[layer])]
        assert [t.data_ptr() for t in attend[1][2:4]] == caches
        assert attend[1][1].data_ptr() == (eng.turned if turn else x[0][layer]).data_ptr() and attend[1][1].shape == (12, 4, 64)
        assert (attend[2]["max_new"] == 9) if cache8 else ("max_new" not in attend[2])
        if turn:   # queries into the engine's own copy: the caller's stay as they are
            assert [t.data_ptr() for t in append[1][-2:]] == [x[0][layer].data_ptr(), eng.turned.data_ptr()]
    assert eng.k_cache.dtype is (torch.float8_e4m3fn if cache8 else torch.bfloat16)


def test_what_does_not_fit_is_refused(serving):
    with pytest.raises(TypeError):
        serving.AttentionEngine(Ctx(), 2, 4, 2, 64, 8, 20, 4, 32, 64, rotation=64)
    with pytest.raises(ValueError):
        serving.AttentionEngine(Ctx(), 2, 4, 2, 64, 8, 20, 4, 32, 64, rotation=_rotation(serving, device=1))
    with pytest.raises(ValueError):
        serving.AttentionEngine(Ctx(), 2, 4, 2, 64, 8, 20, 4, 32, 64, rotation=_rotation(serving, rot_dim=128))
    eng = _engine(serving, True, True)
    with pytest.raises(ValueError):   # more query heads than the engine has room for
        eng.step([1, 1, 0, 0], *_arrays(heads=8))
    assert not serving.calls and eng.cached.tolist() == [0, 0, 0, 0] and len(eng.free) == 20


def test_blocks_of_an_8_bit_cache(serving, monkeypatch):
    """A block's codes take half the bytes of its 16-bit numbers, and a scale per head."""
    made = []
    monkeypatch.setattr(serving, "AttentionEngine", lambda ctx, L, H, Hkv, D, bs, n, *a, **kw: made.append((bs, n)) or 1 / 0)
    room = 64 * 2 * 2 * 2 * 16 * 64 * 2   # 64 blocks of two layers' keys and values, two heads each, of 16 tokens of 64 16-bit numbers
    for cache8, blocks in ((False, 64), (True, room // (2 * 2 * 2 * (16 * 64 + 4)))):
        probe = serving.AttentionProbe(Ctx(), [100], [4], n_layers=2, n_heads=4, n_kv_heads=2, head_dim=64, cache_bytes=room, cache8=cache8)
        with pytest.raises(ZeroDivisionError):
            probe.evaluate(4, 128, 16, True, 1.0)
        assert made.pop() == (16, blocks)
