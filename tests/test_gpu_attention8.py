"""Attention over an 8-bit paged cache (scoot_paged_attention8) against a plain 64-bit form, at the lengths, masks, layouts and
values where it can go wrong, its refusals, and a run of the step's calls together."""
import ctypes

import numpy as np
import pytest

import serving8_ref as R8
import serving_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
F8 = torch.float8_e4m3fn


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


class Batch:
    """Requests of (tokens in the sequence, new ones among them). What no request holds in the cache are the codes that the
    format reserves for NaN, and the scales of blocks that none holds are NaN."""

    def __init__(self, requests, dtype="bf16", H=4, Hkv=2, D=128, bs=16, layout="nhd", seed=0, extra_rows=0, spread=4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.dtype, self.bs, self.H, self.Hkv, self.D = dtype, bs, H, Hkv, D
        self.kv_len = np.array([a for a, _ in requests])
        self.query_start = np.concatenate([[0], np.cumsum([b for _, b in requests])])
        count = -(-self.kv_len // bs)
        nb = int(count.sum()) + 3
        ids = rng.permutation(nb)
        self.table = np.full((len(requests), max(1, int(count.max(initial=0)))), -1)
        held, used, at = torch.zeros((nb, bs), dtype=torch.bool), torch.zeros(nb, dtype=torch.bool), 0
        for r, n in enumerate(count):
            self.table[r, :n] = ids[at:at + n]
            i = np.arange(self.kv_len[r])
            held[self.table[r, i // bs], i % bs] = True
            used[self.table[r, :n]] = True
            at += n
        held, used = held.cuda(), used.cuda()
        self.cache, self.scale = [], []
        for j in range(2):
            x = torch.randn((nb, bs, Hkv, D), generator=g, device="cuda")
            s = torch.exp2(torch.randint(-spread, spread + 1, (nb, Hkv), generator=g, device="cuda").float() - 8)
            if j == 0:
                s = s * 2.0 ** -spread   # keys' scores stay below some tens
            c = (x * 100).clamp(-448, 448).to(F8)
            c.view(torch.uint8)[~held] = 0xFF
            s[~used] = float("nan")
            if layout == "hnd":
                c = c.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(F8)
            self.cache.append(c)
            self.scale.append(s)
        T = int(self.query_start[-1]) + extra_rows
        self.q = torch.randn((T, H, D), generator=g, device="cuda").to(DTYPE[dtype])
        self.factor = D ** -0.5

    def at(self, r, i):
        return int(self.table[r, i // self.bs]), i % self.bs

    def run(self, S, ctx, out=None, lse=None, **kw):
        out = torch.full_like(self.q, 3.0) if out is None else out
        lse = torch.full(self.q.shape[:2], 3.0, device="cuda") if lse is None else lse
        S.scoot_paged_attention8(ctx, self.q, *self.cache, *self.scale, _i32(self.table), _i32(self.query_start), _i32(self.kv_len),
                                 out, self.factor, lse=lse, **kw)
        return out, lse

    def want(self, **kw):
        k, v = (np.nan_to_num(c.contiguous().view(torch.uint8).view(F8).double().cpu().numpy()) for c in self.cache)
        ks, vs = (np.nan_to_num(s.double().cpu().numpy()) for s in self.scale)
        return R8.attention8(self.q.double().cpu().numpy(), k, v, ks, vs, self.table, self.query_start, self.kv_len, self.factor,
                             self.dtype, **kw)

    def check(self, S, ctx, **kw):
        out, lse = self.run(S, ctx, **kw)
        ctx.check()
        self.compare(out, lse, **kw)
        most = int(np.diff(self.query_start).max(initial=0))
        again = self.run(S, ctx, max_new=max(1, most), **kw)
        ctx.check()
        self.compare(*again, **kw)
        return out, lse

    def compare(self, out, lse, **kw):
        T = int(self.query_start[-1])
        o, z, eo, ez = self.want(**kw)
        got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
        empty = np.isneginf(z)[:T]
        assert (got[:T][empty] == 0).all() and np.isneginf(gl[:T][empty]).all()
        assert np.isfinite(got[:T]).all() and np.isfinite(gl[:T][~empty]).all()
        assert (np.abs(got - o)[:T] <= eo[:T]).all(), np.max((np.abs(got - o) / np.maximum(eo, 1e-30))[:T])
        assert (np.abs(gl[:T][~empty] - z[:T][~empty]) <= ez[:T][~empty]).all()
        assert (got[T:] == 3.0).all() and (gl[T:] == 3.0).all()  # rows of no request have no output


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("requests", [
    [(1, 1)], [(2, 2)], [(17, 1)], [(31, 1), (32, 1), (33, 1), (127, 1), (128, 1), (129, 1)], [(5, 5), (128, 128), (131, 3)],
    [(300, 1), (1, 1), (260, 130), (33, 33), (0, 0), (77, 0), (500, 2)], [(400, 300), (700, 1), (290, 257)]])
def test_lengths(S, ctx, dtype, D, requests):
    Batch(requests, dtype=dtype, D=D, seed=D + len(requests), extra_rows=3).check(S, ctx)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (3, 3), (4, 1), (5, 1), (6, 2), (14, 2), (16, 1), (17, 1), (32, 2), (40, 1), (96, 1), (128, 1)])
@pytest.mark.parametrize("requests", [[(70, 1), (200, 1)], [(150, 20), (9, 9), (140, 1)]])
def test_head_groups(S, ctx, H, Hkv, requests):
    Batch(requests, H=H, Hkv=Hkv, D=64 if H % 3 else 128, seed=H).check(S, ctx)


@pytest.mark.parametrize("H,Hkv,most", [(2, 2, 8), (2, 2, 16), (2, 2, 17), (2, 2, 32), (2, 2, 33), (12, 4, 5), (8, 2, 4), (8, 2, 8), (8, 2, 9), (5, 1, 3),
                                        (5, 1, 6), (7, 1, 2), (7, 1, 5), (8, 1, 2), (8, 1, 4), (9, 1, 2), (16, 1, 2), (16, 1, 3)])
@pytest.mark.parametrize("D,dtype,window", [(128, "bf16", 0), (64, "fp16", 0), (64, "bf16", 37)])
def test_a_few_tokens_each(S, ctx, H, Hkv, most, D, dtype, window):
    """With the most that a request brings known: around the numbers of rows at which another kernel or form takes over."""
    requests = [(400, most), (33, 1), (90, max(1, most - 1)), (1500, most), (most, most), (most // 2, most), (0, 0), (257, 2)]
    Batch(requests, dtype=dtype, H=H, Hkv=Hkv, D=D, seed=most + H, extra_rows=2).check(S, ctx, window=window)


@pytest.mark.parametrize("bs", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd"])
@pytest.mark.parametrize("D", [64, 128])
def test_block_sizes_and_layouts(S, ctx, bs, layout, D):
    Batch([(333, 70), (1000, 1), (257, 1), (600, 200)], H=6, Hkv=3, D=D, bs=bs, layout=layout, seed=bs).check(S, ctx)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 7, 33, 128, 200, 5000])
@pytest.mark.parametrize("requests", [[(300, 150), (500, 1), (129, 129), (70, 3)], [(30, 1), (700, 1), (129, 1)], [(900, 400)]])
def test_masks(S, ctx, causal, window, requests):
    Batch(requests, D=64, H=4, Hkv=2, bs=8, seed=window).check(S, ctx, causal=causal, window=window)


def test_rows_that_see_nothing(S, ctx):
    """Tokens before their sequence (more new ones than it has), sequences of none, and a batch of them alone."""
    for requests in ([(3, 10), (0, 5), (200, 1), (0, 0), (40, 300)], [(0, 1), (0, 7)], [(0, 200)], [(1, 400)]):
        Batch(requests, D=64, H=4, Hkv=1, seed=4).check(S, ctx)
    Batch([(3, 10), (0, 5), (40, 300)], D=128, seed=5).check(S, ctx, causal=False, window=2)


@pytest.mark.parametrize("requests", [[(300, 200), (90, 1), (120, 4)], [(50, 3), (64, 2), (700, 9)]])
def test_codes_that_a_token_does_not_see_never_reach_it(S, ctx, requests):
    """Reserved codes among keys and values: tokens before them are as without."""
    b = Batch(requests, D=128, H=4, Hkv=2, seed=19)
    clean = b.run(S, ctx)
    for r, i in ((0, requests[0][0] - 2), (2, requests[2][0] - 1)):
        for c in b.cache:
            c.view(torch.uint8)[b.at(r, i)] = 0x7F
    out, lse = b.run(S, ctx)
    ctx.check()
    sees = torch.zeros(len(out), dtype=torch.bool)
    ends = b.query_start
    sees[ends[1] - 2:ends[1]] = True
    sees[ends[3] - 1] = True
    # (their scores' order of sums does not depend on what is masked)
    assert torch.equal(out[~sees], clean[0][~sees]) and torch.equal(lse[~sees], clean[1][~sees])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_queries_that_are_not_finite_touch_their_row_alone(S, ctx, bad):
    b = Batch([(300, 200), (90, 1), (70, 5)], D=64, H=4, Hkv=2, seed=2)
    clean = b.run(S, ctx)
    for row, head in ((7, 1), (200, 3), (203, 0)):
        b.q[row, head, 11] = bad
    out, lse = b.run(S, ctx)
    ctx.check()
    hit = torch.zeros(out.shape[:2], dtype=torch.bool)
    hit[7, 1] = hit[200, 3] = hit[203, 0] = True
    assert torch.equal(out[~hit], clean[0][~hit]) and torch.equal(lse[~hit], clean[1][~hit])
    assert torch.isnan(out[hit]).all()


def test_large_scores_and_scales(S, ctx):
    """Scores of several hundreds that grow along the sequence, values near the types' ends, and scales far apart."""
    b = Batch([(400, 130), (600, 1), (333, 3)], dtype="bf16", D=64, seed=3)
    b.q *= 30.0
    b.scale[1] *= 2.0 ** 90
    b.check(S, ctx)
    b = Batch([(400, 130), (600, 1)], dtype="fp16", D=128, seed=3, spread=5)
    b.q *= 20.0
    b.check(S, ctx)
    b = Batch([(900, 1), (500, 2), (700, 300)], dtype="bf16", D=128, seed=6)
    for j, low in ((0, 2.0 ** -100), (1, 2.0 ** -60)):   # most blocks' numbers are nothing beside a few blocks'
        b.scale[j][::3] = torch.where(torch.isnan(b.scale[j][::3]), b.scale[j][::3], low)
    b.check(S, ctx)


@pytest.mark.parametrize("dtype,top", [("bf16", 2.0 ** -120), ("bf16", 2.0 ** -14), ("bf16", 2.0 ** 100), ("fp16", 2.0 ** -14), ("fp16", 2.0 ** 10)])
def test_queries_of_any_size(S, ctx, dtype, top):
    b = Batch([(100, 1), (80, 3), (200, 150)], dtype=dtype, D=64, seed=9)
    b.q *= top
    b.factor = float(min(1.0 / top, 2.0 ** 120)) * 64 ** -0.5
    b.check(S, ctx)


def test_scales_of_any_kind(S, ctx):
    """Zeros, and scales that are no powers of two; one that is negative or not finite is flagged and counts as zero."""
    b = Batch([(300, 1), (90, 4), (200, 140)], D=64, seed=7)
    for s in b.scale:
        s *= 1.37
        s[int(b.table[0, 3])] = 0.0
        s[int(b.table[2, 5]), 1] = 0.0
    b.check(S, ctx)
    for bad in (float("nan"), float("inf"), -1.0):
        for j in range(2):
            for r in (0, 2):
                good = b.scale[j][int(b.table[r, 2]), 0].clone()
                b.scale[j][int(b.table[r, 2]), 0] = bad
                out, lse = b.run(S, ctx)
                with pytest.raises(S.ScootError) as e:
                    ctx.check()
                assert e.value.status == -1
                b.scale[j][int(b.table[r, 2]), 0] = 0.0
                b.compare(out, lse)
                b.scale[j][int(b.table[r, 2]), 0] = good
    b.scale[0][:], b.scale[1][:] = 0.0, 0.0   # every score is zero: the mean of zeros
    b.check(S, ctx)


def test_strides(S, ctx):
    """q and out as slices of wider arrays, and a cache whose blocks lie apart."""
    b = Batch([(140, 30), (257, 1), (300, 90)], H=6, Hkv=2, D=64, seed=6)
    T = b.q.shape[0]
    qkv = torch.randn((T, 11, 64), device="cuda").to(b.q.dtype)
    qkv[:, 2:8] = b.q
    wide = torch.full((T, 7, 128), 5.0, device="cuda").to(b.q.dtype)
    for j, c in enumerate(b.cache):
        apart = torch.full((c.shape[0], 2, *c.shape[1:]), 0x7F, dtype=torch.uint8, device="cuda")
        apart[:, 1] = c.view(torch.uint8)
        b.cache[j] = apart[:, 1].view(F8)
    b.q = qkv[:, 2:8]
    out, lse = b.run(S, ctx, out=wide[:, 1:, 64:])
    ctx.check()
    b.compare(out, lse)
    assert (wide[:, :1] == 5.0).all() and (wide[:, :, :64] == 5.0).all()


def test_no_lse(S, ctx):
    b = Batch([(140, 30), (257, 1), (300, 200)], seed=2)
    out, lse = b.run(S, ctx)
    again = torch.empty_like(out)
    S.scoot_paged_attention8(ctx, b.q, *b.cache, *b.scale, _i32(b.table), _i32(b.query_start), _i32(b.kv_len), again, b.factor)
    assert torch.equal(out, again)


def test_offsets_past_32_bits(S, ctx):
    """Blocks whose keys start past 2^32 elements."""
    D, H, bs, nb = 128, 8, 32, (1 << 32) // (128 * 8 * 32) + 700
    b = Batch([(300, 40), (1000, 1)], H=16, Hkv=8, D=D, bs=bs, seed=12)
    n = b.cache[0].shape[0]
    big, scales = [], []
    for c, s in zip(b.cache, b.scale):
        y = torch.empty((nb, bs, H, D), dtype=torch.uint8, device="cuda")
        y[nb - n:] = c.view(torch.uint8)
        z = torch.full((nb, H), float("nan"), device="cuda")
        z[nb - n:] = s
        big.append(y.view(F8))
        scales.append(z)
    out, lse = torch.full_like(b.q, 3.0), torch.full(b.q.shape[:2], 3.0, device="cuda")
    S.scoot_paged_attention8(ctx, b.q, *big, *scales, _i32(b.table + nb - n), _i32(b.query_start), _i32(b.kv_len), out, b.factor, lse=lse)
    ctx.check()
    b.compare(out, lse)


def _torch_want(b, r, chunk=256):
    """(output, sum of p |v|, lse) of request r in 64 bits on the GPU."""
    kv, q0, q1 = int(b.kv_len[r]), int(b.query_start[r]), int(b.query_start[r + 1])
    i = np.arange(kv)
    where = torch.from_numpy(b.table[r][i // b.bs].astype(np.int64)).cuda(), torch.from_numpy(i % b.bs).cuda()
    K, V = (c.view(torch.uint8)[where].view(F8).double() * s[where[0]].double()[..., None] for c, s in zip(b.cache, b.scale))
    parts = []
    for a in range(q0, q1, chunk):
        z = min(q1, a + chunk)
        s = torch.einsum("tgad,kgd->tgak", b.q[a:z].double().unflatten(1, (b.Hkv, -1)), K) * b.factor
        pos = torch.arange(kv - q1 + a, kv - q1 + z, device="cuda")[:, None]
        s = s.masked_fill((torch.arange(kv, device="cuda") > pos)[:, None, None], -float("inf"))
        p = torch.softmax(s, -1)
        parts.append([torch.einsum("tgak,kgd->tgad", p, V).flatten(1, 2), torch.einsum("tgak,kgd->tgad", p, V.abs()).flatten(1, 2),
                      torch.logsumexp(s, -1).flatten(1, 2)])
    return [torch.cat(x) for x in zip(*parts)]


@pytest.mark.parametrize("requests,H,Hkv,D", [
    ("many", 8, 2, 128), ([(50001, 1), (40000, 5)], 8, 1, 128), ([(9000, 700)], 4, 4, 128), ([(30000, 1), (20, 1)], 7, 1, 64),
    ([(5000, 1500), (300, 299), (2500, 1), (100, 1)], 16, 2, 128), ([(6000, 900)], 32, 1, 64), ([(65000, 130)], 4, 1, 128)])
def test_large_batches(S, ctx, requests, H, Hkv, D):
    """Against torch in 64 bits on the GPU: many short sequences, and some that are split over the whole device."""
    if requests == "many":
        requests = [(int(n), 1) for n in np.random.default_rng(3).integers(1, 200, 1500)]
    b = Batch(requests, H=H, Hkv=Hkv, D=D, seed=H)
    out, lse = b.run(S, ctx)
    ctx.check()
    for r in range(0, len(requests), max(1, len(requests) // 300)):
        q0, q1 = int(b.query_start[r]), int(b.query_start[r + 1])
        want, mass, zl = _torch_want(b, r)
        u, f = R.UNIT["bf16"], R.UNIT["fp16"]
        # as serving8_ref.attention8: sum |q k| scale of at most 160 here, scores' roundings 2^-20 of it; a value's least
        # rounding is 2^-32 of its largest code and scale (448 and 2^-4) per key
        tol = u * want.abs() + (f + 2 * 160 * 2.0 ** -20 + 2.0 ** -18) * mass + 2.0 ** -32 * 448 * 2.0 ** -4 * int(b.kv_len[r])
        assert ((out[q0:q1].double() - want).abs() <= tol).all()
        assert ((lse[q0:q1].double() - zl).abs() <= 160 * 2.0 ** -20 + 2.0 ** -17).all()


def test_same_inputs_same_bits(S, ctx):
    b = Batch([(2000, 1), (5000, 1), (700, 300), (90, 90), (4000, 2)], H=8, Hkv=2, D=128, seed=21)
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
        out, lse = torch.empty_like(b.q), torch.empty(b.q.shape[:2], device="cuda")
        args = [_i32(b.table), _i32(b.query_start), _i32(b.kv_len)]
        torch.cuda.synchronize()
        S.scoot_paged_attention8(c2, b.q, *b.cache, *b.scale, *args, out, b.factor, lse=lse, stream=st)
        st.synchronize()
        c2.check()
    assert torch.equal(first[0], out) and torch.equal(first[1], lse)


def test_calls_in_a_row_and_two_graphs_of_one_context(S, ctx):
    """Requests of both kernels and of many parts, each call's outputs taken and overwritten right behind it, and two captured
    graphs over the same workspace and counters replayed in turn."""
    batches = [Batch([(900, 1)] * 40 + [(700, 300), (1500, 700)], H=8, Hkv=2, D=128, seed=31), Batch([(30000, 1), (77, 2), (9000, 40)], H=6, Hkv=2, D=64, seed=32)]
    outs = [(torch.full_like(b.q, 3.0), torch.full(b.q.shape[:2], 3.0, device="cuda")) for b in batches]
    index = [[_i32(b.table), _i32(b.query_start), _i32(b.kv_len)] for b in batches]
    k16 = [torch.randn((4, 16, 2, 128), device="cuda").bfloat16() for _ in range(2)]
    q16, o16, i16 = torch.randn((1, 8, 128), device="cuda").bfloat16(), torch.empty((1, 8, 128), device="cuda").bfloat16(), \
        [_i32([[0, 1, 2, 3]]), _i32([0, 1]), _i32([60])]

    def call(i):
        b, (out, lse) = batches[i], outs[i]
        S.scoot_paged_attention8(ctx, b.q, *b.cache, *b.scale, *index[i], out, b.factor, lse=lse)

    for i in (0, 1, 0):   # (the workspace is there)
        call(i)
    want = [[t.clone() for t in o] for o in outs]
    for o, b in zip(want, batches):
        b.compare(*o)
    taken = []
    for n in range(20):
        call(n % 2)
        taken.append([t.clone() for t in outs[n % 2]])
        for t in outs[n % 2]:
            t.fill_(float("nan"))
        S.scoot_paged_attention(ctx, q16, *k16, *i16, o16, 1.0)
    graphs = [torch.cuda.CUDAGraph() for _ in batches]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i)
    for n in range(20):
        graphs[n % 2].replay()
        taken.append([t.clone() for t in outs[n % 2]])
        for t in outs[n % 2]:
            t.fill_(float("nan"))
    ctx.check()
    for n, got in enumerate(taken):
        assert all(torch.equal(a, b) for a, b in zip(got, want[n % 2])), n


def _step(S, ctx, cached, new, D, H, Hkv, bs, dtype, graphed=False, window=0):
    """Tables, append and attention of a step of an 8-bit cache with rotary positions, and what they should give."""
    rng = np.random.default_rng(len(cached))
    plan = S.Rotation(D)
    width = 12
    R_, T = len(cached), int(new.sum())
    nb = 60
    ids = rng.permutation(nb)
    held = -(-cached // bs)
    table = np.full((R_, width), -1)
    at = 0
    for r in range(R_):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    free = ids[at:]
    g = torch.Generator(device="cuda").manual_seed(5)
    kc, vc = ((torch.randn((nb, bs, Hkv, D), generator=g, device="cuda") * 100).clamp(-448, 448).to(F8) for _ in range(2))
    ks, vs = (torch.exp2(torch.randint(-9, -6, (nb, Hkv), generator=g, device="cuda").float()) for _ in range(2))
    qkv = torch.randn((T, H + 2 * Hkv, D), generator=g, device="cuda").to(DTYPE[dtype])
    q, k, v = qkv.split((H, Hkv, Hkv), 1)
    b = {n: t for n, t in zip(("k", "v", "ks", "vs"), (_codes(kc), _codes(vc), ks.double().cpu().numpy(), vs.double().cpu().numpy()))}
    dev = {"table": _i32(table), "start": torch.zeros(R_ + 1, dtype=torch.int32, device="cuda"), "kv": torch.zeros(R_, dtype=torch.int32, device="cuda"),
           "slot": torch.empty(T, dtype=torch.int64, device="cuda"), "pos": torch.empty(T, dtype=torch.int32, device="cuda"),
           "counts": torch.zeros(2, dtype=torch.int32, device="cuda")}
    turned, out = torch.empty_like(q), torch.empty_like(q)
    c_len, n_len, fr = _i32(cached), _i32(new), _i32(free)

    def call():
        S.scoot_kv_tables(ctx, c_len, n_len, dev["table"], bs, nb, fr, dev["start"], dev["kv"], dev["slot"], dev["pos"], dev["counts"])
        S.scoot_kv_append8(ctx, k, v, dev["slot"], kc, vc, ks, vs, rotation=plan, position=dev["pos"], q=q, q_out=turned)
        S.scoot_paged_attention8(ctx, turned, kc, vc, ks, vs, dev["table"], dev["start"], dev["kv"], out, D ** -0.5, window=window,
                                 max_new=int(new.max()))
    if graphed:
        warm = torch.cuda.Stream()   # (and the workspace is there: lengths are still zero)
        S.scoot_paged_attention8(ctx, q, kc, vc, ks, vs, dev["table"], dev["start"], dev["kv"], out, 1.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=warm):
            call()
        graph.replay()
    else:
        call()
    torch.cuda.synchronize()
    ctx.check()
    tb, start, kv, slot, pos, _ = R.tables(cached, new, table, bs, nb, free, T)
    angle = R8.angles(S.scoot_rotary_turns(S.scoot_rotary_frequencies(D)), pos)
    assert np.array_equal(dev["table"].cpu().numpy(), tb) and np.array_equal(dev["slot"].cpu().numpy(), slot)
    for name, x, cache, scale in (("k", R8.rotate(k.double().cpu().numpy(), angle)[0], kc, ks), ("v", v.double().cpu().numpy(), vc, vs)):
        want_c, want_s = R8.append8(x, slot, b[name], b[name + "s"])
        assert np.array_equal(scale.double().cpu().numpy(), want_s)
        # a rotated number next to a border between two codes may fall on either side
        assert (np.abs(_codes(cache) - want_c) <= np.maximum(2.0 ** -3 * np.abs(want_c), 2.0 ** -9)).all()
    want_q, e = R8.rotate(q.double().cpu().numpy(), angle)
    live = slot >= 0
    tq = turned.double().cpu().numpy()
    assert (np.abs(tq - want_q)[live] <= 1.01 * e[live] + R8.step(dtype, want_q[live])).all()
    o, _, eo, _ = R8.attention8(tq, _codes(kc), _codes(vc), ks.double().cpu().numpy(), vs.double().cpu().numpy(), tb, start, kv, D ** -0.5,
                                dtype, window=window)
    assert (np.abs(out.double().cpu().numpy() - o) <= eo).all()


def _codes(t):
    return t.contiguous().view(torch.uint8).view(F8).double().cpu().numpy()


@pytest.mark.parametrize("D,H,Hkv,bs,dtype,window", [(128, 8, 2, 16, "bf16", 0), (64, 3, 3, 8, "fp16", 20), (128, 7, 1, 32, "fp16", 0)])
@pytest.mark.parametrize("graphed", [False, True])
def test_a_step_of_tables_append_and_attention(S, ctx, D, H, Hkv, bs, dtype, window, graphed):
    _step(S, ctx, np.array([30, 0, 17, 1, 64]), np.array([1, 40, 1, 30, 2]), D, H, Hkv, bs, dtype, graphed, window)
    _step(S, ctx, np.array([30, 5, 17, 1]), np.array([1, 1, 1, 1]), D, H, Hkv, bs, dtype, graphed, window)


@pytest.mark.parametrize("what", ["start falls", "start past", "length", "long", "id", "negative id", "more than said"])
def test_bad_lengths_and_blocks_are_flagged(S, ctx, what):
    b = Batch([(100, 1), (90, 30), (200, 1)], D=64, seed=2)
    kw, skip = {}, []
    if what == "start falls":
        b.query_start[1], skip = 40, [1]
    elif what == "start past":
        b.query_start[3], skip = 999, [2]
    elif what == "length":
        b.kv_len[0], skip = -5, [0]
    elif what == "long":
        b.kv_len[0], skip = b.table.shape[1] * b.bs + 1, [0]
    elif what in ("id", "negative id"):
        b.table[2, 4] = b.cache[0].shape[0] if what == "id" else -2
    else:
        kw, skip = {"max_new": 29}, [1]
    out, lse = b.run(S, ctx, **kw)
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -4
    if what == "start falls":
        return   # its neighbour's tokens are others than were made
    b.query_start[3] = 32
    b.kv_len[0] = max(0, min(int(b.kv_len[0]), 100))
    if what in ("id", "negative id"):   # the block counts as zeros
        b.table[2, 4] = b.table[2, 5]
        for c, s in zip(b.cache, b.scale):
            extra = torch.zeros_like(c.view(torch.uint8)[:1]).view(F8)
            c2 = torch.cat([c.view(torch.uint8), extra.view(torch.uint8)]).view(F8)
            b.cache[0 if c is b.cache[0] else 1] = c2
        b.scale = [torch.cat([s, torch.ones_like(s[:1])]) for s in b.scale]
        b.table[2, 4] = len(b.cache[0]) - 1
    o, z, eo, ez = b.want()
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r in range(3):
        rows = slice(int(b.query_start[r]), int(b.query_start[r + 1]))
        if r in skip:
            assert (got[rows] == 3.0).all() and (gl[rows] == 3.0).all()
        else:
            assert (np.abs(got - o)[rows] <= eo[rows]).all() and (np.abs(gl - z)[rows] <= ez[rows]).all()


def test_refusals(S, ctx):
    b = Batch([(100, 1), (90, 30)], D=64, H=4, Hkv=2, seed=2)
    start, kv, table = _i32(b.query_start), _i32(b.kv_len), _i32(b.table)
    out = torch.empty_like(b.q)
    L, p = S.lib(), lambda t: t.data_ptr()
    lay = S.scoot_kv_layout.from_buffer_copy(S._kv8(*b.cache, *b.scale, b.q.get_device())[0])

    def with_(**kw):
        c = S.scoot_kv_layout.from_buffer_copy(lay)
        for n, v in kw.items():
            setattr(c, n, v)
        return c

    def call(lay=lay, dtype=1, q=p(b.q), ldt=256, ldh=64, H=4, T=31, start=p(start), kv=p(kv), R=2, table=p(table), ld=b.table.shape[1],
             k=p(b.cache[0]), ks=p(b.scale[0]), scale=0.1, window=0, most=0, out=p(out)):
        return L.scoot_paged_attention8(ctx.handle, None if lay is None else ctypes.byref(lay), dtype, q, ldt, ldh, H, T, start, kv, R, table, ld,
                                        k, p(b.cache[1]), ks, p(b.scale[1]), scale, 1, window, most, out, ldt, ldh, None, None)
    INVALID, UNSUPPORTED = -1, -6
    assert call() == 0 and call(T=0, q=None) == 0 and call(R=0, kv=None) == 0
    for kw, status in ((dict(lay=None), INVALID), (dict(lay=with_(dtype=0)), UNSUPPORTED), (dict(lay=with_(head_dim=80)), UNSUPPORTED),
                       (dict(lay=with_(block_size=4)), UNSUPPORTED), (dict(lay=with_(ld_token=136)), INVALID), (dict(lay=with_(n_blocks=0)), INVALID),
                       (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(H=3), INVALID), (dict(H=0), INVALID),
                       (dict(H=258), UNSUPPORTED), (dict(T=-1), INVALID), (dict(T=1 << 31), INVALID), (dict(T=(1 << 29)), INVALID), (dict(R=-1), INVALID),
                       (dict(ld=-1), INVALID), (dict(ld=1 << 30), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
                       (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(window=-1), INVALID), (dict(most=-1), INVALID),
                       (dict(q=None), INVALID), (dict(q=p(b.q) + 2), INVALID), (dict(ldt=252), INVALID), (dict(ldh=32), INVALID), (dict(out=None), INVALID),
                       (dict(start=None), INVALID), (dict(kv=None), INVALID), (dict(table=None), INVALID), (dict(k=None), INVALID),
                       (dict(k=p(b.cache[0]) + 8), INVALID), (dict(ks=None), INVALID), (dict(ks=p(b.scale[0]) + 1), INVALID)):
        assert call(**kw) == status, kw
    ctx.check()
