"""AttentionEngine and AttentionProbe with rotary positions and with an 8-bit cache, against plain 64-bit forms of what each
step appends and attends to."""
import numpy as np
import pytest

import serving8_ref as R8
import serving_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
PLAN = [[30, 0, 17, 1], [1, 40, 1, 0], [1, 1, 33, 9], "finish 2", [1, 1, 50, 1], [0, 0, 0, 0], [16, 1, 1, 3], "finish 0", [64, 1, 1, 1]]


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    from paper_2408_04323_gb300 import scoot as S
    with S.Context(torch.cuda.current_device()) as c:
        yield c


def _values(t):
    if t.dtype is torch.float8_e4m3fn:   # what no token has written may be any code
        return torch.nan_to_num(t.contiguous().view(torch.uint8).view(t.dtype).double()).cpu().numpy()
    return t.double().cpu().numpy()


def _engine(ctx, turn, cache8, dtype="bf16", block=16, window=0, L=2, H=6, Hkv=2, D=64):
    from paper_2408_04323_gb300 import scoot as S
    from paper_2408_04323_gb300.serving import AttentionEngine
    plan = S.Rotation(D // 2, interleaved=block == 8) if turn else None
    return plan, AttentionEngine(ctx, L, H, Hkv, D, block, 40, 4, 96, 200, DTYPE[dtype], window, rotation=plan, cache8=cache8)


def _tokens(gen, L, H, Hkv, D, dtype):
    q = torch.randn((L, 96, H, D), generator=gen, device="cuda").to(DTYPE[dtype])
    k, v = (torch.randn((L, 96, Hkv, D), generator=gen, device="cuda").to(DTYPE[dtype]) for _ in range(2))
    return q, k, v, torch.empty_like(q)


@pytest.mark.parametrize("turn,cache8,dtype,block,window", [(True, False, "bf16", 16, 0), (False, True, "fp16", 8, 20), (True, True, "bf16", 8, 0),
                                                            (True, True, "fp16", 32, 20)])
def test_steps_append_and_attend(ctx, turn, cache8, dtype, block, window):
    from paper_2408_04323_gb300 import scoot as S
    L, H, Hkv, D = 2, 6, 2, 64
    plan, eng = _engine(ctx, turn, cache8, dtype, block, window)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for new in PLAN:
        if isinstance(new, str):
            eng.finish(int(new.split()[1]))
            continue
        q, k, v, out = _tokens(gen, L, H, Hkv, D, dtype)
        asked = q.clone()
        before = [(_values(eng.k_cache[i]), _values(eng.v_cache[i])) + ((_values(eng.k_scale[i]), _values(eng.v_scale[i])) if cache8 else ())
                  for i in range(L)]
        n = eng.step(new, q, k, v, out)
        ctx.check()
        assert n == sum(new) and torch.equal(q, asked)
        slot, pos, table = eng.slot[:n].cpu().numpy(), eng.position[:n].cpu().numpy(), eng.table.cpu().numpy()
        start = np.concatenate([[0], np.cumsum(new)])
        for i in range(L):
            keys, e = _values(k[i, :n]), 0.0
            turned = q[i, :n]
            if turn:
                keys, e = R8.rotate(keys, R8.angles(S.scoot_rotary_turns(S.scoot_rotary_frequencies(D // 2)), pos), interleaved=block == 8)
                turned = torch.empty_like(turned)
                S.scoot_rotary(ctx, plan, q[i, :n], eng.position[:n], turned)
            now = _values(eng.k_cache[i]), _values(eng.v_cache[i])
            if cache8:
                for x, was, s_was, got, s in ((keys, before[i][0], before[i][2], now[0], eng.k_scale[i]), (_values(v[i, :n]), before[i][1], before[i][3], now[1], eng.v_scale[i])):
                    want, s_want = R8.append8(x, slot, was, s_was)
                    assert np.array_equal(_values(s), s_want)
                    # a rotated number next to a border between two codes may fall on either side
                    assert (np.abs(got - want) <= (np.maximum(2.0 ** -3 * np.abs(want), 2.0 ** -9) if turn else 0.0)).all()
                o, _, eo, _ = R8.attention8(_values(turned), *now, _values(eng.k_scale[i]), _values(eng.v_scale[i]), table, start, eng.cached, D ** -0.5,
                                            dtype, window=window)
            else:
                at = now[0].reshape(-1, Hkv, D)[slot]
                assert (np.abs(at - keys) <= 1.01 * e + R8.step(dtype, keys)).all()
                assert np.array_equal(now[1].reshape(-1, Hkv, D)[slot], _values(v[i, :n]))
                o, _, eo, _ = R.attention(_values(turned), *now, table, start, eng.cached, D ** -0.5, window=window, unit=R.UNIT[dtype])
            assert (np.abs(_values(out[i, :n]) - o) <= eo).all()
        if turn:
            assert torch.equal(eng.turned[:n], turned)
    held = sorted(b for row in eng.blocks for b in row)
    assert sorted(held + eng.free) == list(range(40))


@pytest.mark.parametrize("turn,cache8", [(True, False), (False, True), (True, True)])
def test_a_steps_work_may_be_queued_twice(ctx, turn, cache8):
    """As AttentionProbe does when it could not hold the GPU back for long enough."""
    (_, once), (_, twice) = (_engine(ctx, turn, cache8) for _ in range(2))
    for e in (once, twice):
        e.k_cache.view(torch.uint8 if cache8 else torch.int16).zero_()
        e.v_cache.view(torch.uint8 if cache8 else torch.int16).zero_()
    gen = torch.Generator(device="cuda").manual_seed(4)
    for new in ([30, 0, 17, 1], [1, 40, 1, 0], [1, 1, 33, 9]):
        q, k, v, out = _tokens(gen, 2, 6, 2, 64, "bf16")
        k[:, 1::3] *= 8   # scales grow between steps
        other = torch.empty_like(out)
        n = once.step(new, q, k, v, out)
        twice.step(new, q, k, v, other, run=lambda work: (work(), work()))
        ctx.check()
        assert torch.equal(out[:, :n], other[:, :n])
        for name in ("k_cache", "v_cache") + (("k_scale", "v_scale") if cache8 else ()):
            a, b = (getattr(e, name).contiguous() for e in (once, twice))
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_probe_with_an_8_bit_cache(ctx):
    from paper_2408_04323_gb300 import scoot as S
    from paper_2408_04323_gb300.serving import AttentionProbe
    rng = np.random.default_rng(1)
    prompts, outputs = rng.integers(5, 300, 12), rng.integers(1, 9, 12)
    size = dict(n_layers=1, n_heads=8, n_kv_heads=2, head_dim=64, rotation=S.Rotation(64))
    longest = int((prompts + outputs).max())
    room = 2 * 2 * -(-longest // 16) * 16 * 64 * 2 // 4 * 3   # three quarters of the longest request's 16-bit numbers
    assert AttentionProbe(ctx, prompts, outputs, cache_bytes=room, **size).evaluate(8, 512, 16, True, 1.0) is None
    got = AttentionProbe(ctx, prompts, outputs, cache_bytes=room, cache8=True, **size).evaluate(8, 512, 16, True, 1.0)
    assert got is not None and got["ttft"] > 0 and got["throughput"] > 0
    assert got["steps"] >= max(int(outputs.max()), -(-int(prompts.sum()) // 512))
    assert AttentionProbe(ctx, prompts, outputs, cache_bytes=1 << 21, **size).evaluate(8, 512, 16, False)["throughput"] > 0
