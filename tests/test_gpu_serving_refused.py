"""Tables, append and attention together in batches of which the free blocks do not cover all, and with tokens before their
sequence: requests without a key lie among many that have some, so that every block of the attention's grid meets several."""
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


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _step(S, requests, n_free, D, dtype, H=32, Hkv=8, bs=16, **mask):
    """One step of requests [(cached, new)] with n_free free blocks, against the plain forms; returns how many were refused."""
    rng = np.random.default_rng(len(requests) + D)
    cached, new = (np.array([r[i] for r in requests]) for i in (0, 1))
    held, full = -(-cached // bs), -(-(cached + new) // bs)
    n_blocks = int(held.sum()) + n_free + 1
    ids = rng.permutation(n_blocks)
    table = np.full((len(requests), int(full.max())), -1)
    at = 0
    for r, h in enumerate(held):
        table[r, :h] = ids[at:at + h]
        at += h
    free = ids[at:at + n_free]
    T, dt = int(new.sum()), DTYPE[dtype]
    g = torch.Generator(device="cuda").manual_seed(D)
    kc, vc = (torch.randn((n_blocks, bs, Hkv, D), generator=g, device="cuda").to(dt) for _ in range(2))
    q = torch.randn((T, H, D), generator=g, device="cuda").to(dt)
    k, v = (torch.randn((T, Hkv, D), generator=g, device="cuda").to(dt) for _ in range(2))
    out, lse = torch.full_like(q, 3.0), torch.full((T, H), 3.0, device="cuda")
    t = _i32(table)
    start, kv = torch.empty(len(requests) + 1, dtype=torch.int32, device="cuda"), torch.empty(len(requests), dtype=torch.int32, device="cuda")
    slot, pos = torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
    counts = torch.empty(2, dtype=torch.int32, device="cuda")
    with S.Context(torch.cuda.current_device()) as ctx:
        S.scoot_kv_tables(ctx, _i32(cached), _i32(new), t, bs, n_blocks, _i32(free), start, kv, slot, pos, counts)
        S.scoot_kv_append(ctx, k, v, slot, kc, vc)
        S.scoot_paged_attention(ctx, q, kc, vc, t, start, kv, out, D ** -0.5, lse=lse, **mask)
        ctx.check()
    want = R.tables(cached, new, table, bs, n_blocks, free, T)
    for w, x in zip(want, (t, start, kv, slot, pos, counts)):
        assert np.array_equal(w, x.cpu().numpy())
    _compare(q, kc, vc, want[0], want[1], want[2], D, dtype, out, lse, **mask)
    return int(want[-1][1])


def _compare(q, kc, vc, table, start, kv, D, dtype, out, lse, **mask):
    o, z, eo, ez = R.attention(*[x.double().cpu().numpy() for x in (q, kc, vc)], table, start, kv, D ** -0.5, unit=R.UNIT[dtype], **mask)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(z)
    assert empty.any()
    assert (got[empty] == 0).all() and np.isneginf(gl[empty]).all()
    assert (np.abs(got - o) <= eo).all() and (np.abs(gl[~empty] - z[~empty]) <= ez[~empty]).all()


BATCHES = {
    # 249 decodes in their blocks, then a prompt, or a chunk of one, that is refused
    "a refused prompt": ([(64 + 7 * i - (i % 16 == 0), 1) for i in range(249)] + [(0, 512)], 20),
    "a refused chunk": ([(65 + 6 * i, 1) for i in range(100)] + [(777, 700)] + [(65 + 6 * i, 1) for i in range(100)], 9),
    # every 16th decode lacks a block and there is none
    "every 16th": ([(96 if i % 16 == 5 else 100, 1) for i in range(200)], 0),
    "few decodes": ([(100, 1)] * 40 + [(16, 1)] * 2, 0),
    "runs of refusals": ([(300, 1)] * 300 + [(32, 1)] * 300, 0),
    "prompts, half of them refused": ([(33, 90)] * 40, 118),
    "all refused": ([(16, 1)] * 500 + [(0, 300)] * 3, 0),
}


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "fp16")])
@pytest.mark.parametrize("name", BATCHES)
def test_a_step_with_refusals(S, name, D, dtype):
    requests, n_free = BATCHES[name]
    assert _step(S, requests, n_free, D, dtype) > 0


@pytest.mark.parametrize("mask", [{"window": 40}, {"causal": False}])
def test_refusals_under_other_masks(S, mask):
    requests, n_free = BATCHES["a refused chunk"]
    assert _step(S, requests, n_free, 64, "bf16", H=8, Hkv=2, **mask) > 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("requests", [[(300, 3000)], [(0, 1000)] * 3 + [(200, 1)] * 50, [(5, 5), (130, 700), (0, 0), (64, 900)] * 8])
def test_many_tokens_before_their_sequence(S, D, requests):
    """[(tokens in the cache, new tokens)]: the first of a request's new tokens lie before its sequence and see nothing."""
    H, Hkv, bs = 32, 8, 16
    kv = np.array([r[0] for r in requests])
    start = np.concatenate([[0], np.cumsum([r[1] for r in requests])])
    blocks = -(-kv // bs)
    table = np.full((len(requests), max(1, int(blocks.max()))), -1)
    ids, at = np.random.default_rng(D).permutation(int(blocks.sum()) + 1), 0
    for r, n in enumerate(blocks):
        table[r, :n] = ids[at:at + n]
        at += n
    g = torch.Generator(device="cuda").manual_seed(D)
    kc, vc = (torch.randn((len(ids), bs, Hkv, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((int(start[-1]), H, D), generator=g, device="cuda").bfloat16()
    out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device="cuda")
    with S.Context(torch.cuda.current_device()) as ctx:
        S.scoot_paged_attention(ctx, q, kc, vc, _i32(table), _i32(start), _i32(kv), out, D ** -0.5, lse=lse)
        ctx.check()
    _compare(q, kc, vc, table, start, kv, D, "bf16", out, lse)


def test_zeros_go_where_the_strides_say_and_nowhere_else(S):
    """Refused prompts' rows in a slice of a wider output, without and with lse."""
    H, Hkv, D, bs = 12, 2, 64, 16
    kv = np.array([0, 90] * 20)
    new = np.array([70, 1] * 20)
    start = np.concatenate([[0], np.cumsum(new)])
    table = np.full((len(kv), 6), -1)
    table[1::2] = np.random.default_rng(1).permutation(20 * 6).reshape(20, 6)
    g = torch.Generator(device="cuda").manual_seed(5)
    kc, vc = (torch.randn((120, bs, Hkv, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((int(start[-1]), H, D), generator=g, device="cuda").bfloat16()
    wide = torch.full((q.shape[0], H + 2, 2 * D), 5.0, device="cuda", dtype=q.dtype)
    out, again, lse = wide[:, 1:-1, D:], torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device="cuda")
    args = (q, kc, vc, _i32(table), _i32(start), _i32(kv))
    with S.Context(torch.cuda.current_device()) as ctx:
        S.scoot_paged_attention(ctx, *args, out, D ** -0.5)
        S.scoot_paged_attention(ctx, *args, again, D ** -0.5, lse=lse)
        ctx.check()
    assert torch.equal(out, again)
    assert (wide[:, 0] == 5).all() and (wide[:, -1] == 5).all() and (wide[:, :, :D] == 5).all()
    _compare(q, kc, vc, table, start, kv, D, "bf16", again, lse)
