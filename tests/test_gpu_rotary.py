"""Rotary positions (scoot_rotary, scoot_kv_append_rotary) and appends to an 8-bit cache (scoot_kv_append8) against plain 64-bit
forms, at the sizes, places and values where they can go wrong, and their refusals."""
import ctypes

import numpy as np
import pytest

import serving8_ref as R8

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


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _randn(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DTYPE[dtype])


def _angles(S, rot, pos, **kw):
    return R8.angles(S.scoot_rotary_turns(S.scoot_rotary_frequencies(rot, **kw)), pos)


# ---------------------------------------------------------------------------------------------- rotation

@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 16, 16), (3, 5, 64, 64), (17, 8, 128, 128), (200, 3, 80, 48), (77, 28, 64, 32),
                                       (31, 2, 256, 256), (2600, 1, 128, 16), (9, 40, 96, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rotation(S, ctx, T, H, D, rot, interleaved, dtype):
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 1 << 20, T)
    pos[:5] = [0, 1, 2 ** 31 - 1, -1, -2 ** 31][:T]
    x = _randn((T, H, D), dtype, T)
    angle = _angles(S, rot, pos)
    for inverse, magnitude in ((False, 1.0), (True, 1.0), (False, 1.25)):
        plan = S.Rotation(rot, interleaved=interleaved, magnitude=magnitude)
        y = torch.full_like(x, 7.0)
        S.scoot_rotary(ctx, plan, x, _dev(pos), y, inverse=inverse)
        ctx.check()
        want, e = R8.rotate(_np(x), angle, interleaved, magnitude, inverse)
        assert (np.abs(_np(y) - want) <= e * (1 + R8.R.UNIT[dtype]) + R8.step(dtype, want)).all()
        assert torch.equal(y[..., rot:], x[..., rot:])   # what does not turn, bit for bit
        z = x.clone()
        S.scoot_rotary(ctx, plan, z, _dev(pos), z, inverse=inverse)   # in place
        assert torch.equal(y, z)


def test_rotation_strides(S, ctx):
    """Heads in a wider row, and every second token of an output: the rest stays."""
    T, H, D = 61, 3, 64
    wide = _randn((T, 7, 128), "bf16", 1)
    x = wide[:, 2:5, 64:]
    out = torch.full((2 * T, H + 1, D), 9.0, dtype=torch.bfloat16, device="cuda")
    pos = np.arange(T) * 37
    plan = S.Rotation(32, base=500.0)
    S.scoot_rotary(ctx, plan, x, _dev(pos), out[::2, 1:])
    ctx.check()
    want, e = R8.rotate(_np(x), _angles(S, 32, pos, base=500.0))
    assert (np.abs(_np(out[::2, 1:]) - want) <= 1.01 * e + R8.step("bf16", want)).all()
    assert (out[1::2] == 9).all() and (out[:, 0] == 9).all()


def test_gradients(S, ctx):
    """The inverse takes gradients of y to gradients of x: the formula's transpose, and differences of the map itself."""
    T, H, D, rot = 6, 2, 64, 48
    pos = np.array([0, 3, 100, 4097, 131071, 7])
    for interleaved in (False, True):
        plan = S.Rotation(rot, interleaved=interleaved, magnitude=1.2)
        g = _randn((T, H, D), "fp16", 4)
        dx = torch.empty_like(g)
        S.scoot_rotary(ctx, plan, g, _dev(pos), dx, inverse=True)
        angle = _angles(S, rot, pos)
        x = torch.zeros((T, H, D), dtype=torch.float64, requires_grad=True)
        a = torch.from_numpy(angle)[:, None]
        u, v = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
        gu, gv = (lambda z: (z[..., 0:rot:2], z[..., 1:rot:2]) if interleaved else (z[..., :rot // 2], z[..., rot // 2:rot]))(g.double().cpu())
        plan_y = 1.2 * ((u * a.cos() - v * a.sin()) * gu + (v * a.cos() + u * a.sin()) * gv)
        loss = plan_y.sum() + (x[..., rot:] * g.double().cpu()[..., rot:]).sum()
        want = torch.autograd.grad(loss, x)[0].numpy()
        _, e = R8.rotate(_np(g), angle, interleaved, 1.2, True)
        assert (np.abs(_np(dx) - want) <= 1.01 * e + R8.step("fp16", want)).all()
        # differences: the map is linear, so the loss of x + e_i less that of x is its gradient, to the outputs' roundings
        x0 = _randn((T, H, D), "fp16", 5)
        for i in ((0, 0, 3), (4, 1, 40), (3, 0, 60)):
            ys = []
            for delta in (0.0, 1.0):
                xi = x0.clone()
                xi[i] = delta
                y = torch.empty_like(xi)
                S.scoot_rotary(ctx, plan, xi, _dev(pos), y)
                ys.append(_np(y))
            diff = ((ys[1] - ys[0]) * _np(g)).sum()
            # four numbers change, each of them (below 2^3) off by half a step of 2^-11 and by e
            tol = 4 * 2 * (2.0 ** -8 + 2.0 ** -18) * np.abs(_np(g)).max()
            assert abs(diff - want[i]) <= tol


def test_given_frequencies_and_a_stretched_context(S, ctx):
    x = _randn((40, 2, 64), "fp16", 3)
    pos = np.arange(40) * 3331
    f = np.linspace(-2.0, 7.0, 32)
    y = torch.empty_like(x)
    S.scoot_rotary(ctx, S.Rotation(64, frequencies=f), x, _dev(pos), y)
    # against pos * f in fp64: an angle below 2^20 radians is off by 2^-33 there, and the turns by as much
    want, e = R8.rotate(_np(x), pos[:, None] * f)
    assert (np.abs(_np(y) - want) <= 1.01 * e + 1e-8 + R8.step("fp16", want)).all()
    kw = dict(stretch="parts", factor=8.0, low=1.0, high=32.0, original_len=8192)
    S.scoot_rotary(ctx, S.Rotation(64, magnitude=1.2, **kw), x, _dev(pos), y)
    want, e = R8.rotate(_np(x), pos[:, None] * S.scoot_rotary_frequencies(64, **kw), magnitude=1.2)
    assert (np.abs(_np(y) - want) <= 1.01 * e + 1e-8 + R8.step("fp16", want)).all()
    with pytest.raises(ValueError, match="frequencies"):
        S.Rotation(64, frequencies=f[:5])


# ---------------------------------------------------------------------------------------------- appends

def _places(rng, requests, bs, pad=()):
    """Positions and slots of a batch of (cached, new), with tokens without a slot at `pad` (between requests); the number of
    blocks."""
    n_blocks = sum(-(-(c + n) // bs) - c // bs for c, n in requests) + 2
    ids, at, pos, slot = rng.permutation(n_blocks), 0, [], []
    for c, n in requests:
        p = np.arange(c, c + n)
        b = p // bs - c // bs
        slot.append(ids[at + b] * bs + p % bs)
        pos.append(p)
        at += -(-(c + n) // bs) - c // bs
    pos, slot = np.concatenate(pos), np.concatenate(slot)
    for i in pad:
        pos, slot = np.insert(pos, i, 5), np.insert(slot, i, -1)
    return pos, slot, n_blocks


def _cache(shape, layout, dtype, seed):
    nb, bs, h, d = shape
    x = torch.randn(shape if layout == "nhd" else (nb, h, bs, d), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    return x.to(dtype) if layout == "nhd" else x.to(dtype).transpose(1, 2)


REQUESTS = [([(0, 1)], 16, ()), ([(15, 1), (16, 1), (31, 1), (7, 1)], 16, (2,)), ([(5, 70), (0, 8), (3, 1), (100, 33)], 8, (0, 71)),
            ([(1, 600), (255, 3), (256, 256)], 256, ()), ([(i, 1) for i in range(2000)], 32, ()), ([(30, 3000), (0, 31)], 64, (3000,)),
            ([(13, 5000)], 16, ())]


@pytest.mark.parametrize("requests,bs,pad", REQUESTS)
@pytest.mark.parametrize("dtype,D,rot,H,Hkv,layout,interleaved", [
    ("bf16", 128, 128, 8, 2, "nhd", False), ("fp16", 64, 32, 3, 3, "hnd", True), ("bf16", 64, 64, 0, 5, "nhd", True),
    ("fp16", 128, 48, 7, 1, "hnd", False)])
def test_append_with_a_rotation(S, ctx, requests, bs, pad, dtype, D, rot, H, Hkv, layout, interleaved):
    pos, slot, nb = _places(np.random.default_rng(bs), requests, bs, pad)
    T = len(slot)
    qkv = _randn((T, H + 2 * Hkv, D), dtype, T)
    q, k, v = qkv.split((H, Hkv, Hkv), 1)
    kc, vc = (_cache((nb, bs, Hkv, D), layout, DTYPE[dtype], s) for s in (1, 2))
    k0, v0 = kc.clone(), vc.clone()
    out = torch.full((T, H, D), 5.0, dtype=DTYPE[dtype], device="cuda")
    plan = S.Rotation(rot, interleaved=interleaved, magnitude=1.1)
    more = dict(q=q, q_out=out) if H else {}
    S.scoot_kv_append_rotary(ctx, plan, k, v, _dev(slot, np.int64), _dev(pos), kc, vc, **more)
    ctx.check()
    angle = _angles(S, rot, pos)
    live = slot >= 0
    want, e = R8.rotate(_np(k), angle, interleaved, 1.1)
    at = torch.from_numpy(slot[live] // bs).cuda(), torch.from_numpy(slot[live] % bs).cuda()
    got = _np(kc[at])
    assert (np.abs(got - want[live]) <= 1.01 * e[live] + R8.step(dtype, want[live])).all()
    assert torch.equal(vc[at], v[torch.from_numpy(live).cuda()])
    for c, c0 in ((kc, k0), (vc, v0)):   # the other slots stay
        c[at] = c0[at]
        assert torch.equal(c, c0)
    if H:
        want, e = R8.rotate(_np(q), angle, interleaved, 1.1)
        got = _np(out)
        assert (np.abs(got - want)[live] <= 1.01 * e[live] + R8.step(dtype, want[live])).all()
        assert (got[~live] == 5.0).all()


def _codes(t):
    return t.contiguous().view(torch.uint8).view(F8).double().cpu().numpy()


@pytest.mark.parametrize("requests,bs,pad", REQUESTS)
@pytest.mark.parametrize("dtype,D,rot,H,Hkv,layout,interleaved", [
    ("bf16", 128, 128, 8, 2, "nhd", False), ("fp16", 64, 32, 3, 3, "hnd", True), ("bf16", 64, 0, 0, 5, "nhd", False),
    ("fp16", 128, 48, 7, 1, "hnd", False)])
def test_append8(S, ctx, requests, bs, pad, dtype, D, rot, H, Hkv, layout, interleaved):
    """Scales equal, and older codes; new ones within half a step of the numbers that they stand for."""
    pos, slot, nb = _places(np.random.default_rng(bs), requests, bs, pad)
    T = len(slot)
    qkv = _randn((T, H + 2 * Hkv, D), dtype, T)
    qkv *= torch.exp2(torch.arange(T, device="cuda") % 7 - 3).to(qkv.dtype)[:, None, None]   # blocks' numbers differ in size
    q, k, v = qkv.split((H, Hkv, Hkv), 1)
    kc, vc = (_cache((nb, bs, Hkv, D), layout, torch.float32, s).mul_(50).to(F8) for s in (1, 2))
    ks, vs = (torch.exp2(torch.randint(-14, -5, (nb, Hkv), device="cuda").float()) for _ in range(2))
    if layout == "hnd":
        kc, vc = (c.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(F8) for c in (kc, vc))
    before = [_codes(kc), _codes(vc), ks.double().cpu().numpy(), vs.double().cpu().numpy()]
    out = torch.full((T, H, D), 5.0, dtype=DTYPE[dtype], device="cuda")
    more = dict(rotation=S.Rotation(rot, interleaved=interleaved), position=_dev(pos)) if rot else {}
    if H:
        more.update(q=q, q_out=out)
    S.scoot_kv_append8(ctx, k, v, _dev(slot, np.int64), kc, vc, ks, vs, **more)
    ctx.check()
    live = slot >= 0
    kx, ke = R8.rotate(_np(k), _angles(S, rot, pos), interleaved) if rot else (_np(k), 0 * _np(k))
    at = slot[live] // bs, slot[live] % bs
    for x, e, cache, scale, c0, s0 in ((kx, ke, kc, ks, before[0], before[2]), (_np(v), 0 * _np(v), vc, vs, before[1], before[3])):
        want_c, want_s = R8.append8(x, slot, c0, s0)
        got_c, got_s = _codes(cache), scale.double().cpu().numpy()
        assert np.array_equal(got_s, want_s)
        s = got_s[at[0]][:, :, None]
        # half a step of the code (2^-4 of the number, or 2^-10 of the scale), and the rotation's own error
        assert (np.abs(got_c[at] * s - x[live]) <= np.maximum(2.0 ** -4 * np.abs(x[live]), 2.0 ** -10 * s) + 1.07 * e[live]).all()
        got_c[at] = want_c[at] = 0
        assert np.array_equal(got_c, want_c)
    if H:
        want, e = R8.rotate(_np(q), _angles(S, rot, pos), interleaved)
        assert (np.abs(_np(out) - want)[live] <= 1.01 * e[live] + R8.step(dtype, want[live])).all()
        assert (_np(out)[~live] == 5.0).all()


def test_codes_without_a_rotation_are_the_nearest(S, ctx):
    """Every fp16 number of 16 binades, through a scale of one: ties to even, small ones too."""
    x = np.concatenate([np.arange(0, 0x5F01, dtype=np.uint16), np.arange(0x8000, 0xDF01, dtype=np.uint16)]).view(np.float16).astype(np.float64)
    x = np.resize(x, (-(-len(x) // 64), 1, 64))
    x[:, 0, 0] = 448.0
    T = len(x)
    kc, vc = (torch.zeros((T, 8, 1, 64), device="cuda").to(F8) for _ in range(2))
    ks, vs = (torch.full((T, 1), 3e38, device="cuda") for _ in range(2))   # (of blocks that held nothing: not looked at)
    t = torch.from_numpy(x).cuda().half()
    S.scoot_kv_append8(ctx, t, t, _dev(np.arange(T) * 8, np.int64), kc, vc, ks, vs)
    ctx.check()
    assert (ks == 1).all() and (vs == 1).all()
    for c in (kc, vc):
        assert np.array_equal(_codes(c)[:, 0, 0], R8.code_of(x[:, 0]))


def test_scales_at_their_borders(S, ctx):
    """448 times a power of two still fits; the next number does not; zeros and the least numbers get 2^-100; and the
    largest finite ones."""
    one = np.array([448.0, 450.0, 1.75, 1.7578125, 0.0, 2.0 ** -126, 3.0e38, 2.0 ** -95, 447.0])
    x = torch.zeros((9, 1, 64), dtype=torch.bfloat16, device="cuda")
    x[:, 0, 3] = torch.from_numpy(-one).cuda().to(torch.bfloat16)
    kc, vc = (torch.zeros((9, 8, 1, 64), device="cuda").to(F8) for _ in range(2))
    ks, vs = (torch.full((9, 1), float("nan"), device="cuda") for _ in range(2))
    S.scoot_kv_append8(ctx, x, x, _dev(np.arange(9) * 8, np.int64), kc, vc, ks, vs)
    ctx.check()
    want = R8.least_scale(np.abs(_np(x)).max((1, 2)))
    assert np.array_equal(ks[:, 0].double().cpu().numpy(), want) and torch.equal(ks, vs)
    assert want[0] == 1 and want[1] == 2 and want[2] == 2.0 ** -8 and want[3] == 2.0 ** -7 and want[4] == 2.0 ** -100


def test_token_by_token_like_all_at_once(S, ctx):
    """A block filled one token at a time keeps the same scale, and codes within a least step of those of one call."""
    bs, T = 16, 16
    x = _randn((T, 2, 64), "bf16", 8) * torch.exp2(torch.arange(T, device="cuda") - 8.0).to(torch.bfloat16)[:, None, None]
    made = []
    for parts in ([T], [1] * T, [3, 1, 12]):
        kc, vc = (torch.full((3, bs, 2, 64), 0x7F, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
        ks, vs = (torch.full((3, 2), float("nan"), device="cuda") for _ in range(2))
        t = 0
        for n in parts:
            S.scoot_kv_append8(ctx, x[t:t + n], x[t:t + n], _dev(16 + np.arange(t, t + n), np.int64), kc, vc, ks, vs)
            t += n
        ctx.check()
        assert torch.equal(ks[1], vs[1]) and torch.isnan(ks[[0, 2]]).all() and (kc[[0, 2]].view(torch.uint8) == 0x7F).all()
        made.append((_codes(kc)[1], ks[1].double().cpu().numpy()))
    for c, s in made[1:]:
        assert np.array_equal(s, made[0][1])
        # each of up to 15 growths rounds at most once more, by half the least step of its scale: together below 2^-9
        assert (np.abs(c - made[0][0]) <= 2.0 ** -9).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_numbers_that_are_not_finite_are_stored_as_zero_and_flagged(S, ctx, bad):
    x = _randn((3, 2, 128), "bf16", 8)
    y = x.clone()
    y[1, 1, 5] = bad
    x[1, 1, 5] = 0
    got = []
    for k, v in ((x, x), (y, x), (x, y)):
        kc, vc = (torch.zeros((2, 8, 2, 128), device="cuda").to(F8) for _ in range(2))
        ks, vs = (torch.zeros((2, 2), device="cuda") for _ in range(2))
        S.scoot_kv_append8(ctx, k, v, _dev([8, 9, 10], np.int64), kc, vc, ks, vs)
        got.append([_codes(kc), _codes(vc), _np(ks), _np(vs)])
        if k is y or v is y:
            with pytest.raises(S.ScootError) as e:
                ctx.check()
            assert e.value.status == -1
        ctx.check()
    for g in got[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(g, got[0]))


@pytest.mark.parametrize("held", [float("nan"), float("inf"), -1.0])
def test_a_held_scale_that_cannot_be_is_flagged(S, ctx, held):
    x = _randn((1, 1, 64), "fp16", 2)
    kc, vc = (torch.ones((1, 8, 1, 64), device="cuda").to(F8) for _ in range(2))
    ks, vs = (torch.full((1, 1), held, device="cuda") for _ in range(2))
    S.scoot_kv_append8(ctx, x, x, _dev([3], np.int64), kc, vc, ks, vs)
    with pytest.raises(S.ScootError) as e:
        ctx.check()
    assert e.value.status == -1
    c = _codes(kc)[0, :, 0]
    assert (c[:3] == 0).all() and (c[4:] == 1).all() and _np(ks)[0, 0] == R8.least_scale(np.abs(_np(x)).max())


def test_a_held_scale_of_any_size(S, ctx):
    """A zero (of a block of zeros), one that is no power of two, and one that is larger than needed."""
    x = _randn((1, 1, 64), "fp16", 2)
    top = np.abs(_np(x)).max()
    for held in (0.0, 0.3, 2.0 ** -6 * 1.1, 100.0):
        kc, vc = (torch.ones((1, 8, 1, 64), device="cuda").to(F8) for _ in range(2))
        ks, vs = (torch.full((1, 1), held, device="cuda") for _ in range(2))
        h32 = float(ks)
        S.scoot_kv_append8(ctx, x, x, _dev([3], np.int64), kc, vc, ks, vs)
        ctx.check()
        need = R8.least_scale(np.array(top))
        s = max(h32, float(need))
        assert float(ks) == s and float(vs) == s
        c = _codes(kc)[0, :, 0]
        assert (c[:3] == (1.0 if s == h32 else R8.code_of(np.array(np.float32(h32) / need)))).all()
        # a product with 1 / s in fp32 beside the code's own step
        assert (np.abs(c[3] * s - _np(x)[0, 0]) <= np.maximum(2.0 ** -4 * np.abs(_np(x)[0, 0]), 2.0 ** -10 * s) * (1 + 2.0 ** -18)).all()


def test_slots_past_the_cache_are_skipped_and_flagged(S, ctx):
    T, H, D = 40, 2, 64
    x = _randn((T, H, D), "bf16", 1)
    slot = np.arange(T)
    slot[7], slot[20], slot[39] = 64, 1 << 40, -9
    plan, pos = S.Rotation(64), _dev(np.arange(T))
    for eight in (False, True):
        kc, vc = (torch.zeros((8, 8, H, D), device="cuda").to(F8 if eight else torch.bfloat16) for _ in range(2))
        ks, vs = (torch.zeros((8, H), device="cuda") for _ in range(2))
        out = torch.full_like(x, 3.0)
        if eight:
            S.scoot_kv_append8(ctx, x, x, _dev(slot, np.int64), kc, vc, ks, vs, rotation=plan, position=pos, q=x, q_out=out)
        else:
            S.scoot_kv_append_rotary(ctx, plan, x, x, _dev(slot, np.int64), pos, kc, vc, q=x, q_out=out)
        with pytest.raises(S.ScootError) as e:
            ctx.check()
        assert e.value.status == -4
        skipped = [7, 20, 39]
        assert (out[skipped] == 3).all() and not (out[[6, 8, 38]] == 3).all()
        written = (vc.view(torch.uint8) if eight else vc).flatten(0, 1).flatten(1).ne(0).any(1).cpu().numpy()
        assert written.tolist() == [i not in skipped and i < T for i in range(64)]


def test_offsets_past_32_bits(S, ctx):
    """Blocks whose keys start past 2^32 elements, and rows past 2^32 of strided queries."""
    D, H, bs = 128, 8, 32
    nb = (1 << 32) // (bs * H * D) + 3
    x = _randn((2, H, D), "bf16", 3)
    slot, pos = np.array([(nb - 1) * bs - 1, nb * bs - 32]), np.array([5, 6])
    plan = S.Rotation(D)
    want, e = R8.rotate(_np(x), _angles(S, D, pos))
    q = torch.zeros((3, 1 << 32), dtype=torch.bfloat16, device="cuda")
    rows = q[:2, :H * D].unflatten(1, (H, D))
    rows.copy_(x)
    for eight in (False, True):
        kc, vc = (torch.zeros((nb, bs, H, D), dtype=torch.uint8, device="cuda").view(F8) if eight else
                  torch.zeros((nb, bs, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ks, vs = (torch.zeros((nb, H), device="cuda") for _ in range(2))
        out = torch.empty_like(x)
        if eight:
            S.scoot_kv_append8(ctx, x, x, _dev(slot, np.int64), kc, vc, ks, vs, rotation=plan, position=_dev(pos), q=rows, q_out=out)
        else:
            S.scoot_kv_append_rotary(ctx, plan, x, x, _dev(slot, np.int64), _dev(pos), kc, vc, q=rows, q_out=out)
        if eight:  # its block held earlier tokens, by its slot, with a scale of zero
            assert (ks[-2:] > 0).all()
        ctx.check()
        assert (np.abs(_np(out) - want) <= 1.01 * e + R8.step("bf16", want)).all()
        got = torch.stack([vc.view(torch.uint8 if eight else torch.bfloat16)[nb - 2, -1], vc.view(torch.uint8 if eight else torch.bfloat16)[nb - 1, 0]])
        assert (got != 0).any((1, 2)).all()
        del kc, vc


def test_another_stream_and_a_captured_call(S, ctx):
    T, H, D, bs = 300, 4, 64, 16
    x = _randn((T, H, D), "bf16", 1)
    pos, slot, nb = _places(np.random.default_rng(1), [(5, 200), (40, 100)], bs)
    plan, pos, slot = S.Rotation(64), _dev(pos), _dev(slot, np.int64)
    made = []

    def call(c, q, k, kc, vc, ks, vs, out, y, stream=None):
        S.scoot_rotary(c, plan, q, pos, y, stream=stream)
        S.scoot_kv_append8(c, k, k, slot, kc, vc, ks, vs, rotation=plan, position=pos, q=q, q_out=out, stream=stream)

    def state():
        return [*(torch.zeros((nb, bs, H, D), dtype=torch.uint8, device="cuda").view(F8) for _ in range(2)),
                *(torch.zeros((nb, H), device="cuda") for _ in range(2)), torch.empty_like(x), torch.empty_like(x)]
    one, two, three = state(), state(), state()
    call(ctx, x, x, *one)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(ctx, x, x, *two, stream=st)
    torch.cuda.synchronize()
    q, k = torch.zeros_like(x), torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ctx, q, k, *three)
    q.copy_(x), k.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    ctx.check()
    made = [[t.view(torch.uint8) for t in s] for s in (one, two, three)]
    for other in made[1:]:
        assert all(torch.equal(a, b) for a, b in zip(made[0], other))


def test_refusals(S, ctx):
    x = _randn((4, 2, 64), "bf16", 1)
    pos, slot, plan = _dev(np.arange(4)), _dev(np.arange(4), np.int64), S.Rotation(64)
    c16 = [torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c8 = [torch.zeros((2, 8, 2, 64), device="cuda").to(F8) for _ in range(2)]
    sc = [torch.zeros((2, 2), device="cuda") for _ in range(2)]
    L, p = S.lib(), lambda t: t.data_ptr()
    k16, k8 = S.kv_layout(*c16), S.scoot_kv_layout.from_buffer_copy(S._kv8(*c8, *sc, x.get_device())[0])

    def rotary(rot=plan.struct, dtype=1, xp=p(x), ldt=128, ldh=64, H=2, D=64, pos=p(pos), T=4, y=p(x)):
        return L.scoot_rotary(ctx.handle, None if rot is None else ctypes.byref(rot), dtype, xp, ldt, ldh, H, D, pos, T, 0, y, ldt, ldh, None)

    def append(rot=plan.struct, lay=k16, H=2, q=p(x), out=p(x), k=p(x), slot=p(slot), pos=p(pos), T=4, kc=p(c16[0])):
        return L.scoot_kv_append_rotary(ctx.handle, None if lay is None else ctypes.byref(lay), None if rot is None else ctypes.byref(rot),
                                        q, 128, 64, H, out, 128, 64, k, 128, 64, p(x), 128, 64, slot, pos, T, kc, p(c16[1]), None)

    def append8(rot=plan.struct, lay=k8, dtype=1, H=2, q=p(x), out=p(x), k=p(x), slot=p(slot), pos=p(pos), T=4, ks=p(sc[0])):
        return L.scoot_kv_append8(ctx.handle, None if lay is None else ctypes.byref(lay), dtype, None if rot is None else ctypes.byref(rot),
                                  q, 128, 64, H, out, 128, 64, k, 128, 64, p(x), 128, 64, slot, pos, T, p(c8[0]), p(c8[1]), ks, p(sc[1]), None)

    def with_(s, **kw):
        c = type(s).from_buffer_copy(s)
        for n, v in kw.items():
            setattr(c, n, v)
        return c
    INVALID, UNSUPPORTED = -1, -6
    assert rotary() == append() == append8() == 0
    rotations = [(None, INVALID), (with_(plan.struct, turns=None), INVALID), (with_(plan.struct, turns=plan.struct.turns + 4), INVALID),
                 (with_(plan.struct, rot_dim=0), UNSUPPORTED), (with_(plan.struct, rot_dim=24), UNSUPPORTED), (with_(plan.struct, rot_dim=80), INVALID),
                 (with_(plan.struct, magnitude=float("nan")), INVALID), (with_(plan.struct, magnitude=float("inf")), INVALID)]
    for rot, status in rotations:
        assert rotary(rot=rot) == status and append(rot=rot) == status
        assert append8(rot=rot) == status
    for kw, status in ((dict(dtype=2), UNSUPPORTED), (dict(D=0), UNSUPPORTED), (dict(D=72), UNSUPPORTED), (dict(D=272), UNSUPPORTED),
                       (dict(T=-1), INVALID), (dict(T=1 << 31), INVALID), (dict(H=0), INVALID), (dict(xp=None), INVALID), (dict(y=None), INVALID),
                       (dict(xp=p(x) + 2), INVALID), (dict(ldt=60), INVALID), (dict(ldh=65), INVALID), (dict(pos=None), INVALID)):
        assert rotary(**kw) == status, kw
    for call, lay in ((append, k16), (append8, k8)):
        for kw, status in ((dict(lay=None), INVALID), (dict(lay=with_(lay, head_dim=96)), UNSUPPORTED), (dict(lay=with_(lay, block_size=12)), UNSUPPORTED),
                           (dict(lay=with_(lay, n_blocks=0)), INVALID), (dict(lay=with_(lay, dtype=7)), UNSUPPORTED), (dict(H=-1), INVALID),
                           (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(k=None), INVALID), (dict(slot=None), INVALID), (dict(pos=None), INVALID),
                           (dict(T=-1), INVALID)):
            assert call(**kw) == status, (call, kw)
        assert call(T=0, q=None, k=None, slot=None) == 0
    assert append(lay=with_(k16, dtype=2)) == UNSUPPORTED and append8(lay=with_(k8, dtype=1)) == UNSUPPORTED
    assert append8(dtype=2) == UNSUPPORTED and append8(ks=None) == INVALID and append8(ks=p(sc[0]) + 2) == INVALID
    assert append8(lay=with_(k8, ld_head=72)) == INVALID and append8(rot=None, H=0, pos=None, q=None, out=None) == 0
    ctx.check()
