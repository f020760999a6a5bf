"""Rotary frequencies on the host, the plain forms that the GPU tests compare with, and what the binding of rotary positions and
of the 8-bit cache passes on and refuses (no GPU)."""
import ctypes

import numpy as np
import pytest

import serving8_ref as R8
from test_serving_binding import BF16, I32, S, Tensor, _context, lib  # noqa: F401

torch = pytest.importorskip("torch")
F8, F32, I64 = torch.float8_e4m3fn, torch.float32, torch.int64


# ---------------------------------------------------------------------------------------------- frequencies

@pytest.mark.parametrize("d,base", [(16, 10000.0), (64, 500000.0), (128, 10000.0), (2, 7.0)])
def test_frequencies(S, d, base):
    i = np.arange(d // 2)
    f = base ** (-2.0 * i / d)
    # a power and a quotient or two in fp64: a few units of 2^-53, times the logarithm of the base
    tol = 2.0 ** -48
    assert np.allclose(S.scoot_rotary_frequencies(d, base), f, rtol=tol, atol=0)
    assert np.allclose(S.scoot_rotary_frequencies(d, base, "linear", 4.0), f / 4, rtol=tol, atol=0)
    if d > 2:
        g = S.scoot_rotary_frequencies(d, base, "base", 4.0)
        assert g[0] == 1.0 and np.isclose(g[-1], f[-1] / 4, rtol=tol, atol=0) and (g[1:] < f[1:]).all()
    g = S.scoot_rotary_frequencies(d, base, "parts", 8.0, low=1.0, high=32.0, original_len=4096)
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(g[turns >= 32], f[turns >= 32], rtol=tol, atol=0) and np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=tol, atol=0)
    mid = (turns > 1) & (turns < 32)
    assert ((g[mid] < f[mid]) & (g[mid] > f[mid] / 8)).all()


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=7), dict(base=0.0), dict(base=float("nan")), dict(base=float("inf")),
                                 dict(stretch="linear", factor=0.0), dict(stretch="base", factor=-1.0), dict(stretch="base", rot_dim=2, factor=2.0),
                                 dict(stretch="parts", factor=2.0), dict(stretch="parts", factor=2.0, original_len=100, low=3.0, high=3.0)])
def test_frequencies_that_cannot_be(S, bad):
    with pytest.raises(S.ScootError):
        S.scoot_rotary_frequencies(**{"rot_dim": 64, **bad})


def test_turns(S):
    f = np.array([2 * np.pi * 0.25, 2 * np.pi * 3.5, -2 * np.pi * 0.125, 0.0, 1.0, 1e-4, -1e-9])
    t = S.scoot_rotary_turns(f)
    # a quotient in fp64, and what is below 2^-64
    for x, got in zip(f, t.tolist()):
        want = x / (2 * np.pi) % 1.0
        off = abs(got * 2.0 ** -64 - want)
        assert min(off, 1 - off) <= 2.0 ** -52 * abs(x / (2 * np.pi)) + 2.0 ** -63
    for bad in (np.array([1.0, np.nan]), np.array([np.inf]), np.array([])):
        with pytest.raises(S.ScootError):
            S.scoot_rotary_turns(bad)
    with pytest.raises(ValueError, match="stretch"):
        S.scoot_rotary_frequencies(64, stretch="longer")


# ---------------------------------------------------------------------------------------------- plain forms by hand

def test_plain_rotation_by_hand():
    x = np.array([[[1.0, 0.0, 0.0, 2.0, 5.0]]])
    a = np.array([[np.pi / 2, 0.0]])
    assert np.allclose(R8.rotate(x, a)[0][0, 0], [0.0, 0.0, 1.0, 2.0, 5.0])
    assert np.allclose(R8.rotate(x, a, interleaved=True)[0][0, 0], [0.0, 1.0, 0.0, 2.0, 5.0])
    assert np.allclose(R8.rotate(x, a, magnitude=3.0, inverse=True)[0][0, 0], [0.0, 0.0, -3.0, 6.0, 5.0])
    assert np.allclose(R8.angles(np.array([1 << 62, (1 << 64) - 1], np.uint64), np.array([3, -2])) / R8.TURN, [[-0.25, 0.0], [-0.5, 0.0]])


def test_plain_codes_by_hand():
    assert len(R8.CODES) == 127 and R8.CODES[126] == 448 and R8.CODES[1] == 2.0 ** -9 and (np.diff(R8.CODES) > 0).all()
    got = torch.arange(127, dtype=torch.uint8).view(F8).double().numpy()
    assert (got == R8.CODES).all()
    assert R8.code_of(np.array([1.0625, 1.1875, -1.0626, 500.0, 2.0 ** -10, 3 * 2.0 ** -10])).tolist() == [1.0, 1.25, -1.125, 448.0, 0.0, 2.0 ** -8]
    assert R8.least_scale(np.array([448.0, 448.1, 0.0, 1.75, 1e-40])).tolist() == [1.0, 2.0, 2.0 ** -100, 2.0 ** -8, 2.0 ** -100]
    # a block of 8 with two tokens of scale 1; two new ones that need 4
    cache, scale = np.zeros((1, 8, 1, 1)), np.ones((1, 1))
    cache[0, :2, 0, 0] = [448.0, 2.0 ** -8]
    c, s = R8.append8(np.array([[[1000.0]], [[-3.0]]]), np.array([2, 3]), cache, scale)
    assert s[0, 0] == 4 and c[0, :5, 0, 0].tolist() == [112.0, 0.0, 256.0, -0.75, 0.0]


# ---------------------------------------------------------------------------------------------- the library and its binding

def test_a_missing_context_is_an_error_code(S):
    L, n = S.lib(), None
    assert L.scoot_rotary(n, n, 0, n, 0, 0, 1, 64, n, 1, 0, n, 0, 0, n) == -1
    assert L.scoot_kv_append_rotary(n, n, n, n, 0, 0, 0, n, 0, 0, n, 0, 0, n, 0, 0, n, n, 1, n, n, n) == -1
    assert L.scoot_kv_append8(n, n, 0, n, n, 0, 0, 0, n, 0, 0, n, 0, 0, n, 0, 0, n, n, 1, n, n, n, n, n) == -1
    assert L.scoot_paged_attention8(n, n, 0, n, 0, 0, 1, 0, n, n, 0, n, 0, n, n, n, n, 1.0, 1, 0, 0, n, 0, 0, n, n) == -1


def _rotation(S, device=0):
    r = object.__new__(S.Rotation)   # without a GPU there is none to be had
    r.device, r.struct = device, S.scoot_rotation(4096, 64, 0, 1.0, 0)
    r.ref = ctypes.byref(r.struct)
    return r


def _rotary(S, ctx=None, change={}, device=0, **kw):
    a = {"x": Tensor((4, 2, 64), BF16), "position": Tensor((4,), I32), "out": Tensor((4, 2, 64), BF16), **change}
    S.scoot_rotary(ctx, _rotation(S, device), a["x"], a["position"], a["out"], **kw)


def _append(S, ctx=None, change={}, device=0, **kw):
    a = {"k": Tensor((4, 2, 64), BF16), "v": Tensor((4, 2, 64), BF16), "slot": Tensor((4,), I64), "position": Tensor((4,), I32),
         "k_cache": Tensor((8, 16, 2, 64), BF16), "v_cache": Tensor((8, 16, 2, 64), BF16), "q": Tensor((4, 6, 64), BF16),
         "q_out": Tensor((4, 6, 64), BF16), **change}
    S.scoot_kv_append_rotary(ctx, _rotation(S, device), **a, **kw)


CACHE8 = {"k_cache": ((8, 16, 2, 64), F8), "v_cache": ((8, 16, 2, 64), F8), "k_scale": ((8, 2), F32), "v_scale": ((8, 2), F32)}


def _append8(S, ctx=None, change={}, device=0, **kw):
    a = {"k": Tensor((4, 2, 64), BF16), "v": Tensor((4, 2, 64), BF16), "slot": Tensor((4,), I64), "position": Tensor((4,), I32),
         "q": Tensor((4, 6, 64), BF16), "q_out": Tensor((4, 6, 64), BF16)} | {n: Tensor(*t) for n, t in CACHE8.items()} | change
    S.scoot_kv_append8(ctx, rotation=_rotation(S, device), **a, **kw)


def _attention8(S, ctx=None, change={}, device=0, **kw):
    a = {"q": Tensor((4, 6, 64), BF16), "out": Tensor((4, 6, 64), BF16), "block_table": Tensor((2, 5), I32),
         "query_start": Tensor((3,), I32), "kv_len": Tensor((2,), I32)} | {n: Tensor(*t) for n, t in CACHE8.items()} | change
    S.scoot_paged_attention8(ctx, **a, scale=0.125, **kw)


NEW = {n: ((4, 2, 64), BF16) for n in "kv"} | {n: ((4, 6, 64), BF16) for n in ("q", "q_out")} | {"slot": ((4,), I64), "position": ((4,), I32)}
CALLS = {"rotary": (_rotary, {"x": ((4, 2, 64), BF16), "out": ((4, 2, 64), BF16), "position": ((4,), I32)}),
         "append": (_append, NEW | {n: ((8, 16, 2, 64), BF16) for n in ("k_cache", "v_cache")}),
         "append8": (_append8, NEW | CACHE8),
         "attention8": (_attention8, {n: ((4, 6, 64), BF16) for n in ("q", "out")} | CACHE8 |
                        {"block_table": ((2, 5), I32), "query_start": ((3,), I32), "kv_len": ((2,), I32)})}


@pytest.mark.parametrize("name", CALLS)
def test_a_tensor_on_another_device_is_refused(S, lib, name):
    call, tensors = CALLS[name]
    for ctx in (_context(S, 0), None):
        call(S, ctx)
        for which, (shape, dtype) in tensors.items():
            with pytest.raises(ValueError, match="device"):
                call(S, ctx, change={which: Tensor(shape, dtype, device=1)})
    with pytest.raises(ValueError, match="device"):
        call(S, _context(S, 1))
    if name != "attention8":
        with pytest.raises(ValueError, match="rotation"):
            call(S, device=1)
    assert len(lib.calls) == 2


@pytest.mark.parametrize("name", CALLS)
def test_host_memory_and_other_types_are_refused(S, lib, name):
    call, tensors = CALLS[name]
    for which, (shape, dtype) in tensors.items():
        with pytest.raises(TypeError, match="CUDA"):
            call(S, None, change={which: torch.zeros(shape, dtype=dtype)})
        with pytest.raises(TypeError):
            call(S, None, change={which: Tensor(shape, torch.float64)})
    assert not lib.calls


@pytest.mark.parametrize("name", CALLS)
def test_shapes_that_do_not_match_are_refused(S, lib, name):
    call, tensors = CALLS[name]
    for which, (shape, dtype) in tensors.items():
        if which in ("block_table",):
            continue
        with pytest.raises(ValueError):
            call(S, None, change={which: Tensor((shape[0] + 1, *shape[1:]), dtype)})
    assert not lib.calls


def test_what_comes_together(S, lib):
    for call in (_append, _append8):
        with pytest.raises(ValueError, match="together"):
            call(S, change={"q": None})
        with pytest.raises(ValueError, match="position"):
            call(S, change={"position": None})
        call(S, change={"q": None, "q_out": None})
    a = {n: Tensor(*t) for n, t in (NEW | CACHE8).items() if n not in ("q", "q_out", "position")}
    S.scoot_kv_append8(None, **a)
    with pytest.raises(ValueError, match="rotation"):
        S.scoot_kv_append8(None, **a, position=Tensor((4,), I32))
    with pytest.raises(TypeError, match="Rotation"):
        S.scoot_kv_append8(None, **a, position=Tensor((4,), I32), rotation=3)
    assert len(lib.calls) == 3


@pytest.mark.parametrize("given,passed", [(0, 0), (7, 7), (2 ** 32 + 5, 2 ** 31 - 1), (-2 ** 32 + 5, -1)])
def test_ints_beyond_32_bits_are_not_small_ones(S, lib, given, passed):
    _attention8(S, window=given)
    _attention8(S, max_new=given)
    assert lib.calls[0][19] == passed and lib.calls[1][20] == passed


def test_the_default_stream_is_the_devices_current_one(S, lib):
    for call, _ in CALLS.values():
        call(S, _context(S, 0))
        assert lib.calls[-1][-1] == 1000
