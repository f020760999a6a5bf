"""What the binding of a serving step's calls passes to the library, and what it refuses, with tensors and a library that only
record (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def S():
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot
    return scoot


class Tensor:
    """As much of a contiguous CUDA tensor as the binding asks for."""
    is_cuda = True

    def __init__(self, shape, dtype, device=0):
        self.shape, self.dtype, self.device_index = torch.Size(shape), dtype, device

    def stride(self):
        out, n = [], 1
        for s in reversed(self.shape):
            out.append(n)
            n *= s
        return tuple(reversed(out))

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)


class Library:
    """Takes the calls' arguments as ctypes would pass them; every call succeeds."""

    def __init__(self, S):
        self.protos, self.calls = S._PROTOS, []

    def __getattr__(self, name):
        def call(*args):
            types = self.protos[name]
            assert len(args) == len(types)
            self.calls.append([t(a).value if t in (ctypes.c_int32, ctypes.c_int64) else a for t, a in zip(types, args)])
            return 0
        return call


@pytest.fixture()
def lib(S, monkeypatch):
    L = Library(S)
    monkeypatch.setattr(S, "lib", lambda: L)
    monkeypatch.setattr(S, "_current_stream", lambda device: 1000 + device)
    return L


I32, BF16 = torch.int32, torch.bfloat16


def _attention(S, ctx=None, T=4, R=2, change={}, **kw):
    a = {"q": Tensor((T, 4, 64), BF16), "k_cache": Tensor((8, 16, 2, 64), BF16), "v_cache": Tensor((8, 16, 2, 64), BF16),
         "block_table": Tensor((R, 5), I32), "query_start": Tensor((R + 1,), I32), "kv_len": Tensor((R,), I32),
         "out": Tensor((T, 4, 64), BF16), **change}
    S.scoot_paged_attention(ctx, *a.values(), 0.125, **kw)


def _tables(S, ctx=None, bs=16, R=2, T=4, change={}, **kw):
    a = {"cached_len": Tensor((R,), I32), "new_len": Tensor((R,), I32), "block_table": Tensor((R, 5), I32), "bs": bs, "n_blocks": 8,
         "free_blocks": Tensor((3,), I32), "query_start": Tensor((R + 1,), I32), "kv_len": Tensor((R,), I32),
         "slot": Tensor((T,), torch.int64), "position": Tensor((T,), I32), "counts": Tensor((2,), I32), **change}
    S.scoot_kv_tables(ctx, *a.values(), **kw)


@pytest.mark.parametrize("window,passed", [(0, 0), (7, 7), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1),
                                           (-1, -1), (-2 ** 32 + 5, -1)])
def test_a_window_beyond_32_bits_is_not_a_small_one(S, lib, window, passed):
    _attention(S, window=window)
    assert lib.calls[0][16] == passed


@pytest.mark.parametrize("bs,passed", [(16, 16), (2 ** 32 + 16, 2 ** 31 - 1), (-2 ** 32 + 16, -1)])
def test_a_block_size_beyond_32_bits_is_not_a_small_one(S, lib, bs, passed):
    _tables(S, bs=bs)
    assert lib.calls[0][4] == passed


def test_requests_beyond_32_bits_are_not_a_few(S, lib):
    with pytest.raises(ValueError):
        _tables(S, R=2 ** 32 + 2)
    _attention(S, R=2 ** 32 + 2)
    assert lib.calls[0][9] == 2 ** 31 - 1   # which the library refuses


def _append(S, ctx=None, change={}, **kw):
    a = {"k": Tensor((4, 2, 64), BF16), "v": Tensor((4, 2, 64), BF16), "slot": Tensor((4,), torch.int64),
         "k_cache": Tensor((8, 16, 2, 64), BF16), "v_cache": Tensor((8, 16, 2, 64), BF16), **change}
    S.scoot_kv_append(ctx, *a.values(), **kw)


def _context(S, device):
    ctx = object.__new__(S.Context)   # without a GPU there is none to be had
    ctx.device, ctx.handle = device, None
    return ctx


CALLS = {"tables": (_tables, {n: ((2,), I32) for n in ("cached_len", "new_len", "kv_len", "counts")} |
                    {"block_table": ((2, 5), I32), "free_blocks": ((3,), I32), "query_start": ((3,), I32),
                     "slot": ((4,), torch.int64), "position": ((4,), I32)}),
         "append": (_append, {n: ((4, 2, 64), BF16) for n in "kv"} | {n: ((8, 16, 2, 64), BF16) for n in ("k_cache", "v_cache")} |
                    {"slot": ((4,), torch.int64)}),
         "attention": (_attention, {n: ((4, 4, 64), BF16) for n in ("q", "out")} |
                       {n: ((8, 16, 2, 64), BF16) for n in ("k_cache", "v_cache")} |
                       {"block_table": ((2, 5), I32), "query_start": ((3,), I32), "kv_len": ((2,), I32)})}


@pytest.mark.parametrize("name", CALLS)
def test_a_tensor_on_another_device_than_the_contexts_is_refused(S, lib, name):
    call, tensors = CALLS[name]
    for ctx in (_context(S, 0), None):   # a bare handle's device is that of the call's first array
        call(S, ctx)
        for which, (shape, dtype) in tensors.items():
            with pytest.raises(ValueError, match="device"):
                call(S, ctx, change={which: Tensor(shape, dtype, device=1)})
    with pytest.raises(ValueError, match="device"):
        call(S, _context(S, 1))
    assert len(lib.calls) == 2


def test_a_lse_on_another_device_is_refused(S, lib):
    _attention(S, lse=Tensor((4, 4), torch.float32))
    with pytest.raises(ValueError, match="lse"):
        _attention(S, lse=Tensor((4, 4), torch.float32, device=1))
    assert len(lib.calls) == 1


@pytest.mark.parametrize("name", CALLS)
def test_host_memory_is_refused(S, lib, name):
    call, tensors = CALLS[name]
    host = {which: torch.zeros(shape, dtype=dtype) for which, (shape, dtype) in tensors.items()}
    for ctx in (_context(S, 0), None):
        for which, t in host.items():
            with pytest.raises(TypeError, match="CUDA"):
                call(S, ctx, change={which: t})
        with pytest.raises(TypeError, match="CUDA"):
            call(S, ctx, change=host)
    if name != "tables":
        with pytest.raises(TypeError, match="CUDA"):
            S.kv_layout(host["k_cache"], host["v_cache"])
    assert not lib.calls


def test_the_default_stream_is_the_devices_current_one(S, lib):
    for device, ctx in ((0, _context(S, 0)), (0, None)):
        for call, at in ((_tables, 16), (_append, 12), (_attention, 21)):
            call(S, ctx)
            assert lib.calls[-1][at] == 1000 + device
