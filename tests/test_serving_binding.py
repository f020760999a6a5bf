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
