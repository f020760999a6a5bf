"""A serving step's operators (scoot_kv_tables, scoot_kv_append, scoot_paged_attention) against plain 64-bit forms, at the
lengths, masks, layouts and strides where they can go wrong, and their refusals."""
import ctypes

import numpy as np
import pytest

import serving_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot
    return scoot


@pytest.fixture()
def ctx(S):
    with S.Context(torch.cuda.current_device()) as c:
        yield c


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


# ---------------------------------------------------------------------------------------------- tables

def _run_tables(S, ctx, cached, new, table, bs, n_blocks, free, n_tokens):
    n = len(cached)
    t = _i32(table)
    out = (torch.full((n + 1,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda"),
           torch.full((n_tokens,), -7, dtype=torch.int64, device="cuda"),
           torch.full((n_tokens,), -7, dtype=torch.int32, device="cuda"), torch.full((2,), -7, dtype=torch.int32, device="cuda"))
    S.scoot_kv_tables(ctx, _i32(cached), _i32(new), t, bs, n_blocks, _i32(free), *out)
    return [x.cpu().numpy() for x in (t, *out)]


def _case(rng, n, bs, c_hi, n_hi, zero=0.0):
    cached, new = rng.integers(0, c_hi + 1, n), rng.integers(0, n_hi + 1, n)
    new[rng.random(n) < zero] = 0
    held, full = -(-cached // bs), -(-(cached + new) // bs)
    n_blocks = int(full.sum()) + 5
    ids = rng.permutation(n_blocks)
    table = np.full((n, max(1, int(full.max(initial=0)))), -1)
    at = 0
    for r in range(n):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    return cached, new, table, n_blocks, ids[at:]


@pytest.mark.parametrize("n,bs,c_hi,n_hi,zero", [
    (1, 16, 0, 1, 0.0), (1, 8, 33, 0, 0.0), (2, 256, 300, 700, 0.0), (33, 8, 100, 1, 0.0), (57, 16, 48, 40, 0.5),
    (300, 32, 64, 3, 0.2), (1025, 16, 40, 2, 0.1), (3001, 8, 30, 20, 0.3), (7, 64, 0, 4099, 0.0), (26001, 8, 20, 3, 0.3)])
@pytest.mark.parametrize("pad", [0, 13])
def test_tables_match_the_plain_form(S, ctx, n, bs, c_hi, n_hi, zero, pad):
    cached, new, table, n_blocks, free = _case(np.random.default_rng(n * 100 + bs), n, bs, c_hi, n_hi, zero)
    T = int(new.sum()) + pad
    want = R.tables(cached, new, table, bs, n_blocks, free, T)
    got = _run_tables(S, ctx, cached, new, table, bs, n_blocks, free, T)
    for w, g in zip(want, got):
        assert np.array_equal(w, g)
    ctx.check()


@pytest.mark.parametrize("free_share", [0.0, 0.4, 0.9])
def test_tables_refuse_what_the_free_blocks_do_not_cover(S, ctx, free_share):
    cached, new, table, n_blocks, free = _case(np.random.default_rng(5), 200, 8, 40, 30, 0.2)
    need = int((-(-(cached + new) // 8) + -cached // 8).sum())
    free = free[:int(need * free_share)]
    T = int(new.sum())
    want = R.tables(cached, new, table, 8, n_blocks, free, T)
    assert want[-1][1] > 0
    got = _run_tables(S, ctx, cached, new, table, 8, n_blocks, free, T)
    for w, g in zip(want, got):
        assert np.array_equal(w, g)
    ctx.check()  # refusing is no error


def test_tables_of_no_request_and_of_no_token(S, ctx):
    got = _run_tables(S, ctx, [], [], np.zeros((0, 4)), 16, 10, [1, 2], 3)
    assert got[1].tolist() == [0] and got[3].tolist() == [-1] * 3 and got[4].tolist() == [0] * 3 and got[5].tolist() == [0, 0]
    got = _run_tables(S, ctx, [5, 0], [0, 0], np.array([[3], [-1]]), 16, 10, [1, 2], 0)
    assert got[1].tolist() == [0, 0, 0] and got[2].tolist() == [5, 0] and got[5].tolist() == [0, 0]
    ctx.check()


@pytest.mark.parametrize("what", ["cached", "new", "long", "held id", "free id", "tokens"])
def test_tables_flag_bad_values(S, ctx, what):
    cached, new, table, n_blocks, free = _case(np.random.default_rng(8), 20, 8, 30, 12)
    cached[3], new[3], table[3, 0], T = 5, 6, 0, int(new.sum()) - int(new[3]) + 6
    if what == "cached":
        cached[3] = -1
    elif what == "new":
        new[3] = -2
    elif what == "long":
        cached[3] = table.shape[1] * 8
    elif what == "held id":
        table[3, 0] = n_blocks
    elif what == "free id":
        free = free.copy()
        free[0] = -3
    else:
        T -= 4
    want = R.tables(cached, new, table, 8, n_blocks, free, T)
    got = _run_tables(S, ctx, cached, new, table, 8, n_blocks, free, T)
    for w, g in zip(want, got):
        assert np.array_equal(w, g)
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -4
    ctx.check()


def test_tables_flag_a_length_beyond_32_bits(S, ctx):
    """Rows wide enough for 2^31 tokens: the longest length is served, and one more token refused."""
    bs, width = 256, (1 << 23) + 1
    table = torch.zeros((2, width), dtype=torch.int32, device="cuda")
    longest = 2 ** 31 - 1
    out = {k: torch.full((n,), -7, dtype=t, device="cuda") for k, n, t in
           (("query_start", 3, torch.int32), ("kv_len", 2, torch.int32), ("slot", 2, torch.int64), ("position", 2, torch.int32),
            ("counts", 2, torch.int32))}
    S.scoot_kv_tables(ctx, _i32([longest - 1, longest]), _i32([1, 1]), table, bs, 4, _i32([]), out["query_start"], out["kv_len"],
                      out["slot"], out["position"], out["counts"])
    assert out["query_start"].tolist() == [0, 1, 2] and out["counts"].tolist() == [0, 1]
    assert out["kv_len"].tolist() == [longest, 0]
    assert out["position"].tolist() == [longest - 1, longest] and out["slot"].tolist() == [(longest - 1) % bs, -1]
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -4


# ---------------------------------------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,H,D,bs,layout", [(1, 1, 64, 8, "nhd"), (7, 3, 128, 16, "hnd"), (513, 8, 128, 32, "nhd"),
                                             (2049, 5, 64, 16, "hnd"), (100, 12, 64, 256, "nhd")])
def test_append_writes_its_slots_and_nothing_else(S, ctx, dtype, T, H, D, bs, layout):
    g = torch.Generator(device="cuda").manual_seed(T)
    nb = -(-T // bs) + 3
    shape = (nb, bs, H, D) if layout == "nhd" else (nb, H, bs, D)
    kc, vc = (torch.randn(shape, generator=g, device="cuda").to(DTYPE[dtype]) for _ in range(2))
    if layout == "hnd":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    qkv = torch.randn((T, 2 * H + 3, D), generator=g, device="cuda").to(DTYPE[dtype])
    k, v = qkv[:, 1:1 + H], qkv[:, 2 + H:2 + 2 * H]
    slot = torch.randperm(nb * bs, generator=g, device="cuda")[:T]
    slot[T // 2] = -1
    want = [kc.clone(), vc.clone()]
    live = slot >= 0
    for w, x in zip(want, (k, v)):
        w[slot[live] // bs, slot[live] % bs] = x[live]
    S.scoot_kv_append(ctx, k, v, slot, kc, vc)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])
    ctx.check()


def test_append_flags_a_slot_past_the_cache_and_skips_it(S, ctx):
    kc, vc = torch.zeros((4, 8, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 8, 2, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    S.scoot_kv_append(ctx, k, k, torch.tensor([32, 31], device="cuda"), kc, vc)
    assert float(kc.float().sum()) == 128 and float(kc[3, 7].float().sum()) == 128 and torch.equal(kc, vc)
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -4


# ---------------------------------------------------------------------------------------------- attention

class Batch:
    """A batch of requests ((tokens in the sequence, new tokens), ...) over a cache whose blocks lie in no order; slots
    that hold no token are NaN in keys and values."""

    def __init__(self, requests, dtype="bf16", H=4, Hkv=2, D=64, bs=16, layout="nhd", seed=0, extra_rows=0, fill=float("nan")):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        dt = DTYPE[dtype]
        self.dtype, self.bs = dtype, bs
        self.kv_len = np.array([a for a, _ in requests], np.int32)
        self.query_start = np.concatenate([[0], np.cumsum([b for _, b in requests])]).astype(np.int32)
        n_blocks = int(sum(-(-a // bs) for a, _ in requests)) + 3
        ids = rng.permutation(n_blocks)
        self.table = np.full((len(requests), int(max(-(-a // bs) for a, _ in requests)) + 1), n_blocks + 5, np.int32)
        shape = (n_blocks, bs, Hkv, D) if layout == "nhd" else (n_blocks, Hkv, bs, D)
        k, v = (torch.randn(shape, generator=g, device="cuda").to(dt) for _ in range(2))
        self.k, self.v = (k, v) if layout == "nhd" else (k.transpose(1, 2), v.transpose(1, 2))
        held = torch.zeros((n_blocks, bs), dtype=torch.bool)
        at = 0
        for r, (a, _) in enumerate(requests):
            n = -(-a // bs)
            self.table[r, :n] = ids[at:at + n]
            i = np.arange(a)
            held[self.table[r, i // bs], i % bs] = True
            at += n
        free = ~held.cuda()
        self.k[free] = fill
        self.v[free] = fill
        T = int(self.query_start[-1]) + extra_rows
        self.q = torch.randn((T, H, D), generator=g, device="cuda").to(dt)
        self.scale = D ** -0.5

    def at(self, r, i):
        return int(self.table[r, i // self.bs]), i % self.bs

    def run(self, S, ctx, out=None, lse=None, **kw):
        out = torch.full_like(self.q, 3.0) if out is None else out
        lse = torch.full(self.q.shape[:2], 3.0, device="cuda") if lse is None else lse
        S.scoot_paged_attention(ctx, self.q, self.k, self.v, _i32(self.table), _i32(self.query_start), _i32(self.kv_len),
                                out, self.scale, lse=lse, **kw)
        return out, lse

    def want(self, **kw):
        f = [x.double().cpu().numpy() for x in (self.q, self.k, self.v)]
        with np.errstate(invalid="ignore"):
            return R.attention(*f, self.table, self.query_start, self.kv_len, self.scale, unit=R.UNIT[self.dtype], **kw)

    def check(self, S, ctx, **kw):
        out, lse = self.run(S, ctx, **kw)
        ctx.check()
        self.compare(out, lse, **kw)
        return out, lse

    def compare(self, out, lse, **kw):
        T = int(self.query_start[-1])
        o, z, eo, ez = self.want(**kw)
        got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
        empty = np.isneginf(z)[:T]
        assert (got[:T][empty] == 0).all() and np.isneginf(gl[:T][empty]).all()
        assert np.isfinite(got[:T]).all() and np.isfinite(gl[:T][~empty]).all()
        assert (np.abs(got - o)[:T] <= eo[:T]).all(), np.max((np.abs(got - o) / np.maximum(eo, 1e-30))[:T])
        assert (np.abs(gl - z)[:T][~empty] <= ez[:T][~empty]).all()
        assert (got[T:] == 3.0).all() and (gl[T:] == 3.0).all()  # rows of no request have no output


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("requests", [
    [(1, 1)], [(2, 2)], [(17, 1)], [(127, 1), (128, 1), (129, 1)], [(5, 5), (128, 128), (131, 3)],
    [(300, 1), (1, 1), (260, 130), (33, 33), (0, 0), (77, 0), (500, 2)]])
def test_attention_lengths(S, ctx, dtype, D, requests):
    Batch(requests, dtype=dtype, D=D, seed=D + len(requests), extra_rows=3).check(S, ctx)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (4, 1), (5, 1), (6, 2), (14, 2), (16, 1), (32, 2), (40, 1), (96, 1), (128, 1)])
@pytest.mark.parametrize("requests", [[(70, 1), (200, 1)], [(150, 20), (9, 9), (140, 1)]])
def test_attention_head_groups(S, ctx, H, Hkv, requests):
    Batch(requests, H=H, Hkv=Hkv, D=64 if H % 3 else 128, seed=H).check(S, ctx)


@pytest.mark.parametrize("bs", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd"])
def test_attention_block_sizes_and_layouts(S, ctx, bs, layout):
    Batch([(259, 3), (130, 130), (513, 1)], dtype="fp16", bs=bs, layout=layout, D=128, seed=bs).check(S, ctx)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 2, 37, 128, 129, 5000])
def test_attention_masks(S, ctx, causal, window):
    Batch([(300, 70), (40, 40), (290, 1), (1, 1)], H=4, Hkv=2, seed=window).check(S, ctx, causal=causal, window=window)


def test_attention_rows_that_see_nothing(S, ctx):
    b = Batch([(3, 3), (200, 150), (40, 1)], seed=4)
    b.kv_len = np.array([0, 100, 40], np.int32)  # a refused request, and one whose first 50 tokens lie before its start
    b.check(S, ctx)
    b.check(S, ctx, causal=False)
    b.check(S, ctx, window=8)


@pytest.mark.parametrize("requests", [[(400, 300)], [(150, 1)], [(700, 1)], [(260, 20), (300, 90)]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_token_does_not_see_never_reaches_it(S, ctx, requests, bad):
    """Values that are not finite at keys outside the window of every row, and at keys that only later rows see."""
    b = Batch(requests, D=128, seed=9, fill=bad)
    window = 40
    n = int(b.query_start[1])
    first = int(b.kv_len[0]) - n
    hide = [i for i in range(max(0, first - window + 1))][-3:]
    if n > 2:
        hide.append(first + n - 1)  # only the last row sees it
    for i in hide:
        b.v[b.at(0, i)] = bad
        b.k[b.at(0, i)] = bad
    out, lse = b.run(S, ctx, window=window)
    ctx.check()
    o, z, eo, ez = b.want(window=window)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    rows = np.ones(len(got), bool)
    if n > 2:
        rows[n - 1] = False
    assert np.isfinite(got[rows]).all()
    assert (np.abs(got - o)[rows] <= eo[rows]).all() and (np.abs(gl - z)[rows] <= ez[rows]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_values_that_a_token_sees_do_reach_it(S, ctx, bad):
    """A value that is not finite reaches the rows that see its key, in its dimension, and no other."""
    b = Batch([(300, 200), (90, 1)], D=128, H=4, Hkv=2, seed=19)
    b.v[b.at(0, 180)][..., 1, 5] = bad  # key 180 is seen by rows 80 on; key-value head 1
    out, _ = b.run(S, ctx)
    got = out.double().cpu().numpy()
    reach = np.zeros(got.shape, bool)
    reach[80:200, 2:, 5] = True
    assert np.isfinite(got[~reach]).all()
    assert np.isnan(got[reach]).all() if bad != bad else (got[reach] == bad).all()


def test_large_scores_and_values(S, ctx):
    """Scores of several hundreds (one key takes nearly all), growing along the sequence, and values near the type's end."""
    b = Batch([(400, 130), (600, 1), (333, 7)], dtype="bf16", D=64, seed=3)
    b.k *= torch.linspace(1, 60, b.k.shape[0], device="cuda").to(b.k.dtype)[:, None, None, None]
    b.v *= 1e30
    b.check(S, ctx)
    b = Batch([(400, 130), (600, 1)], dtype="fp16", D=128, seed=3)
    b.q *= 20.0
    b.v *= 1000.0
    b.check(S, ctx)


def test_attention_strides(S, ctx):
    """q and out as slices of wider arrays, and a cache whose blocks lie apart."""
    b = Batch([(140, 30), (257, 1)], H=6, Hkv=2, D=64, seed=6)
    T = b.q.shape[0]
    qkv = torch.randn((T, 11, 64), device="cuda").to(b.q.dtype)
    qkv[:, 2:8] = b.q
    wide = torch.full((T, 7, 128), 5.0, device="cuda").to(b.q.dtype)
    for name in ("k", "v"):
        x = getattr(b, name)
        apart = torch.full((x.shape[0], 2, *x.shape[1:]), float("nan"), device="cuda").to(x.dtype)
        apart[:, 1] = x
        setattr(b, name, apart[:, 1])
    b.q = qkv[:, 2:8]
    out = wide[:, 1:, 64:]
    out, lse = b.run(S, ctx, out=out)
    ctx.check()
    b.compare(out, lse)
    assert (wide[:, :1] == 5.0).all() and (wide[:, :, :64] == 5.0).all()


def test_no_lse(S, ctx):
    b = Batch([(140, 30), (257, 1)], seed=2)
    out, lse = b.run(S, ctx)
    again = torch.empty_like(out)
    S.scoot_paged_attention(ctx, b.q, b.k, b.v, _i32(b.table), _i32(b.query_start), _i32(b.kv_len), again, b.scale)
    assert torch.equal(out, again)


def test_offsets_past_32_bits(S, ctx):
    """Blocks whose keys start past 2^32 elements."""
    D, H, bs, n_blocks = 128, 8, 32, (1 << 32) // (128 * 8 * 32) + 700
    b = Batch([(300, 40), (1000, 1)], H=16, Hkv=8, D=D, bs=bs, seed=12)
    big = []
    for x in (b.k, b.v):
        y = torch.empty((n_blocks, bs, H, D), dtype=x.dtype, device="cuda")
        y[n_blocks - x.shape[0]:] = x
        big.append(y)
    table = np.where(b.table < b.k.shape[0], b.table + n_blocks - b.k.shape[0], n_blocks)
    out, lse = torch.full_like(b.q, 3.0), torch.full(b.q.shape[:2], 3.0, device="cuda")
    S.scoot_paged_attention(ctx, b.q, *big, _i32(table), _i32(b.query_start), _i32(b.kv_len), out, b.scale, lse=lse)
    ctx.check()
    b.compare(out, lse)
    slot = torch.tensor([n_blocks * bs - 1], device="cuda")
    x = torch.full((1, H, D), 7.0, device="cuda", dtype=b.q.dtype)
    S.scoot_kv_append(ctx, x, x, slot, *big)
    ctx.check()
    assert (big[0][-1, -1] == 7).all() and (big[1][-1, -1] == 7).all()


def test_a_large_batch_of_single_tokens_and_a_long_sequence(S, ctx):
    """Against torch in 64 bits on the GPU: many short sequences, and one that is split over the whole device."""
    rng = np.random.default_rng(3)
    for requests, H, Hkv in (([(int(n), 1) for n in rng.integers(1, 200, 1500)], 8, 2), ([(50001, 1), (40000, 5)], 8, 1),
                             ([(9000, 700)], 4, 4)):
        b = Batch(requests, H=H, Hkv=Hkv, D=128, seed=H)
        out, lse = b.run(S, ctx)
        ctx.check()
        G = H // Hkv
        for r, (kv, n) in enumerate(requests):
            q0 = int(b.query_start[r])
            i = np.arange(kv)
            where = torch.from_numpy(b.table[r][i // b.bs].astype(np.int64)).cuda(), torch.from_numpy(i % b.bs).cuda()
            K, V = b.k[where].double(), b.v[where].double()
            s = torch.einsum("tgad,kgd->tgak", b.q[q0:q0 + n].double().reshape(n, Hkv, G, 128), K) * b.scale
            hidden = torch.arange(kv, device="cuda") > torch.arange(kv - n, kv, device="cuda")[:, None]
            s = s.masked_fill(hidden[:, None, None], -float("inf"))
            p = torch.softmax(s, -1)
            want = torch.einsum("tgak,kgd->tgad", p, V).reshape(n, H, 128)
            mass = torch.einsum("tgak,kgd->tgad", p, V.abs()).reshape(n, H, 128)
            u = R.UNIT["bf16"]
            # as serving_ref.attention: scores of at most 12 here, 2^-20 of sum |q k| scale <= 40
            tol = u * want.abs() + (u + 2 * 40 * 2.0 ** -20 + 2.0 ** -18) * mass + 1e-6
            assert ((out[q0:q0 + n].double() - want).abs() <= tol).all()
            zl = torch.logsumexp(s, -1).reshape(n, H)
            assert ((lse[q0:q0 + n].double() - zl).abs() <= 40 * 2.0 ** -20 + 2.0 ** -17).all()


def test_same_inputs_same_bits(S, ctx):
    b = Batch([(2000, 1), (5000, 1), (700, 300), (90, 90)], H=8, Hkv=2, D=128, seed=21)
    first = b.run(S, ctx)
    for _ in range(5):
        again = b.run(S, ctx)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_another_stream_and_another_context(S, ctx):
    b = Batch([(900, 1), (300, 150)], H=8, Hkv=2, D=128, seed=22)
    first = b.run(S, ctx)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with S.Context(torch.cuda.current_device()) as c2:
        out, lse = torch.empty_like(first[0]), torch.empty_like(first[1])
        args = (_i32(b.table), _i32(b.query_start), _i32(b.kv_len))
        torch.cuda.synchronize()
        S.scoot_paged_attention(c2, b.q, b.k, b.v, *args, out, b.scale, lse=lse, stream=st)
        st.synchronize()
        assert torch.equal(first[0], out) and torch.equal(first[1], lse)


def test_a_captured_step_follows_its_lengths(S, ctx):
    """tables, append and attention in one graph, replayed with other lengths and values in the same buffers."""
    H, Hkv, D, bs, n_blocks, width, n_req, T = 8, 2, 64, 16, 200, 40, 5, 64
    dev = dict(device="cuda")
    cached, new, kv_len = (torch.zeros(n_req, dtype=torch.int32, **dev) for _ in range(3))
    table = torch.full((n_req, width), -1, dtype=torch.int32, **dev)
    free = torch.zeros(n_blocks, dtype=torch.int32, **dev)
    start, counts = torch.zeros(n_req + 1, dtype=torch.int32, **dev), torch.zeros(2, dtype=torch.int32, **dev)
    slot, pos = torch.zeros(T, dtype=torch.int64, **dev), torch.zeros(T, dtype=torch.int32, **dev)
    q = torch.zeros((T, H, D), dtype=torch.bfloat16, **dev)
    k, v = (torch.zeros((T, Hkv, D), dtype=torch.bfloat16, **dev) for _ in range(2))
    kc, vc = (torch.zeros((n_blocks, bs, Hkv, D), dtype=torch.bfloat16, **dev) for _ in range(2))
    out = torch.zeros_like(q)

    def step(st=None):
        S.scoot_kv_tables(ctx, cached, new, table, bs, n_blocks, free, start, kv_len, slot, pos, counts, stream=st)
        S.scoot_kv_append(ctx, k, v, slot, kc, vc, stream=st)
        S.scoot_paged_attention(ctx, q, kc, vc, table, start, kv_len, out, D ** -0.5, stream=st)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = np.random.default_rng(1)
    have, used = np.zeros(n_req, int), 0
    K, V = [np.zeros((0, Hkv, D))] * n_req, [np.zeros((0, Hkv, D))] * n_req
    free_ids = rng.permutation(n_blocks)
    for i in range(4):
        n = rng.integers(0, 13, n_req)
        cached.copy_(_i32(have))
        new.copy_(_i32(n))
        free.copy_(_i32(np.roll(free_ids, -used)))
        for x in (q, k, v):
            x.normal_()
        out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        ctx.check()
        used += int(counts[0])
        assert int(counts[1]) == 0
        at = np.concatenate([[0], np.cumsum(n)])
        for r in range(n_req):
            K[r] = np.concatenate([K[r], k[at[r]:at[r + 1]].double().cpu().numpy()])
            V[r] = np.concatenate([V[r], v[at[r]:at[r + 1]].double().cpu().numpy()])
        have += n
        width_t = max(1, int(have.max()))  # a table of one block per request
        kc2, vc2 = (np.zeros((n_req, width_t, Hkv, D)) for _ in range(2))
        for r in range(n_req):
            kc2[r, :have[r]], vc2[r, :have[r]] = K[r], V[r]
        o, _, eo, _ = R.attention(q.double().cpu().numpy(), kc2, vc2, np.arange(n_req)[:, None], at, have, D ** -0.5)
        got = out.double().cpu().numpy()
        assert (np.abs(got - o)[:at[-1]] <= eo[:at[-1]]).all()


# ---------------------------------------------------------------------------------------------- refusals

@pytest.mark.parametrize("what", ["table", "kv long", "kv negative", "starts", "start past"])
def test_attention_flags_bad_values(S, ctx, what):
    b = Batch([(100, 1), (60, 8), (30, 2)], seed=1)
    if what == "table":
        b.table[1, 1] = b.k.shape[0]
    elif what == "kv long":
        b.kv_len[1] = b.table.shape[1] * b.bs + 1
    elif what == "kv negative":
        b.kv_len[1] = -4
    elif what == "starts":
        b.query_start[1] = 10
    else:
        b.query_start[-1] = b.q.shape[0] + 1
    out, _ = b.run(S, ctx)
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -4
    if what in ("table", "kv long", "kv negative"):  # the other requests are as they were
        good = Batch([(100, 1), (60, 8), (30, 2)], seed=1).run(S, ctx)[0]
        assert torch.equal(out[0], good[0]) and torch.equal(out[9:], good[9:])
    if what.startswith("kv"):
        assert (out[1:9] == 3.0).all()
    ctx.check()


def test_attention_refuses_bad_arguments(S, ctx):
    b = Batch([(100, 4)], seed=1)
    args = [b.q, b.k, b.v, _i32(b.table), _i32(b.query_start), _i32(b.kv_len), torch.empty_like(b.q), b.scale]

    def status(i=None, x=None, **kw):
        a = list(args)
        if i is not None:
            a[i] = x
        try:
            S.scoot_paged_attention(ctx, *a, **kw)
        except S.ScootError as e:
            return e.status
        except (TypeError, ValueError) as e:
            return type(e)
        return 0

    assert status() == 0
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert status(7, bad) == -1
    assert status(window=-1) == -1
    assert status(0, b.q.float()) is TypeError
    assert status(0, b.q.cpu()) is TypeError
    assert status(0, b.q[:, :, ::2]) is ValueError
    assert status(6, b.q[:3]) is ValueError
    assert status(4, _i32([0, 4, 4])) is ValueError
    assert status(5, _i32(b.kv_len).long()) in (TypeError, ValueError)
    assert status(2, b.v.half()) is TypeError
    odd = torch.empty(b.q.numel() + 1, dtype=b.q.dtype, device="cuda")[1:].view(b.q.shape)
    assert status(0, odd) == -1  # not 16-byte aligned
    tight = torch.empty((4, 4, 68), dtype=b.q.dtype, device="cuda")[..., :64]
    assert status(0, tight) == -1  # a stride that is no multiple of 8
    assert status(0, b.q[:, :3].contiguous()) is ValueError
    x = torch.empty((4, 3, 64), dtype=b.q.dtype, device="cuda")
    a = list(args)
    a[0], a[6] = x, x.clone()
    with pytest.raises(S.ScootError) as e:  # 3 heads over 2
        S.scoot_paged_attention(ctx, *a)
    assert e.value.status == -1
    for shape in ((4, 12, 2, 64), (4, 4, 2, 64), (4, 512, 2, 64), (4, 16, 2, 96)):  # block sizes and a head size
        c = torch.empty(shape, dtype=b.q.dtype, device="cuda")
        a = list(args)
        a[0] = torch.empty((4, 4, shape[3]), dtype=b.q.dtype, device="cuda")
        a[6] = a[0].clone()
        a[1] = a[2] = c
        with pytest.raises(S.ScootError) as e:
            S.scoot_paged_attention(ctx, *a)
        assert e.value.status == -6
    c = torch.empty((4, 16, 1, 64), dtype=b.q.dtype, device="cuda")
    x = torch.empty((4, 129, 64), dtype=b.q.dtype, device="cuda")
    with pytest.raises(S.ScootError) as e:
        S.scoot_paged_attention(ctx, x, c, c, *args[3:6], x.clone(), b.scale)
    assert e.value.status == -6
    ctx.check()


def test_attention_refuses_more_requests_than_its_sums_hold(S, ctx):
    """By the C entry point, whose check of the sizes comes before that of the (missing) arrays."""
    b = Batch([(100, 4)], seed=1)
    ref = S._kv(b.k, b.v)[1]

    def message(n_req):
        status = S.lib().scoot_paged_attention(S._h(ctx), ref, None, 512, 128, 4, 4, None, None, n_req, None, 8, b.k.data_ptr(),
                                               b.v.data_ptr(), 1.0, 1, 0, None, 512, 128, None, None)
        with pytest.raises(S.ScootError) as e:
            S._check(status, "scoot_paged_attention", S._h(ctx))
        assert e.value.status == -1
        return str(e.value)

    assert "n_req" in message(2 ** 30 + 1) and "n_req" in message(-1)
    assert "q is NULL" in message(2 ** 30)
    ctx.check()


def test_nothing_to_do_is_no_error(S, ctx):
    b = Batch([(100, 4)], seed=1)
    none = torch.empty((0, 4, 64), dtype=b.q.dtype, device="cuda")
    S.scoot_paged_attention(ctx, none, b.k, b.v, _i32(b.table), _i32([0, 0]), _i32(b.kv_len), none.clone(), b.scale)
    S.scoot_paged_attention(ctx, b.q, b.k, b.v, _i32(b.table[:0]), _i32([0]), _i32([]), torch.empty_like(b.q), b.scale)
    S.scoot_kv_append(ctx, none[:, :2], none[:, :2], torch.empty(0, dtype=torch.int64, device="cuda"), b.k, b.v)
    ctx.check()
