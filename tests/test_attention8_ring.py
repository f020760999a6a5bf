"""The waits between the roles of the paged attention's kernel over a cache of codes, as a model on the CPU: no order of the roles
may leave all of them waiting, no wait for a parity may meet a barrier that is two phases away from it, and no place in the rings
of scales and exponents may be taken again before all have read it.

Beside the roles of the kernel's other form: four warps that make the tiles of keys and values in place of the copies, one of which
writes the tile's scales, and with bf16 a warp per slot that turns its queries.  While it waits for queries the product warp
issues the products that get ready."""
import random
import re
from collections import deque

import pytest

import test_attention_ring as T

SCALES = dict(zip((128, 64), map(int, re.search(r"kScaleRing = D == 128 \? (\d+) : (\d+)", T.TEXT).groups())))
UPS = T.number("kUpRing")
LESS = dict(((128, 0), (64, int(re.search(r"- \(k8 && D == 64 \? (\d+) : 0\)", T.TEXT).group(1)))))
WARPS, TURN_READS = 4, 4


def looks_at_products_while_queries_come():
    """Whether the product warp issues what gets ready while it waits for queries."""
    scores = T.TEXT[T.TEXT.index("auto scores = [&]"):]
    return re.search(r"ready\(q_bar, q_phase\); \+\+i\) \{\s*if \(n_todo && ready\(p_bar\(\), p_phase\(\)\)\) values\(\);",
                     scores[:scores.index("wait.at(q_bar, q_phase)")]) is not None


class Places:
    """A ring's places: what each holds, and how many are still to read it."""

    def __init__(self, n):
        self.at = [(None, 0)] * n

    def write(self, i, readers):
        assert self.at[i % len(self.at)][1] == 0, "taken again before it was read"
        self.at[i % len(self.at)] = (i, readers)

    def read(self, i):
        held, left = self.at[i % len(self.at)]
        assert held == i and left > 0, "not what was written"
        self.at[i % len(self.at)] = (held, left - 1)


def run(items, D, rng, turn, looks):
    """One CTA's items (units, pair) through the roles in a random order; raises T.Stall if all wait."""
    ns, kbuf = T.STAGES[D] - LESS[D], T.BUFS[D]
    listed, at = [], 0
    for nu, pair in items:
        listed.append((nu, 2 if pair else at))
        if not pair:
            at ^= 1
    full = [T.Barrier() for _ in range(T.RING)]
    empty = [T.Barrier(2 + 1 + WARPS + (2 if turn else 0)) for _ in range(T.RING)]  # (softmax as a whole, products, codes, queries)
    kv_full, kv_empty = [T.Barrier(WARPS) for _ in range(ns)], [T.Barrier() for _ in range(ns)]
    q_full, q_ready, q_empty = ([T.Barrier(), T.Barrier()] for _ in range(3))
    s_full, p_full, pv_done = ([[T.Barrier() for _ in range(3)] for _ in range(2)] for _ in range(3))
    ring = [None] * T.RING
    copies, tensor = [], deque()
    scales, ups = Places(SCALES[D]), [Places(UPS), Places(UPS)]

    def item_warp():
        n_q = [0, 0]
        for k, it in enumerate(listed + [None]):
            if k >= T.RING:
                yield lambda: empty[k % T.RING].passed(k // T.RING - 1)
            ring[k % T.RING] = it
            full[k % T.RING].arrive()
            for s in (0, 1):
                if it and it[1] in (s, 2):
                    if n_q[s]:
                        yield lambda: q_empty[s].passed(n_q[s] - 1)
                    copies.append(q_full[s])
                    n_q[s] += 1

    def code_warp(w):
        at = unit = k = 0
        while True:
            yield lambda: full[k % T.RING].passed(k // T.RING)
            it = ring[k % T.RING]
            if it is None:
                return
            empty[k % T.RING].arrive()
            for n in range(2 * it[0]):
                if at >= ns:
                    yield lambda: kv_empty[at % ns].passed(at // ns - 1)
                else:
                    yield None
                if w == 0 and n % 2 == 0:
                    scales.write(unit, 2 if it[1] == 2 else 1)
                    unit += 1
                kv_full[at % ns].arrive()
                at += 1
            k += 1

    def turn_warp(s):
        n_q = k = 0
        while True:
            yield lambda: full[k % T.RING].passed(k // T.RING)
            it = ring[k % T.RING]
            if it is None:
                return
            empty[k % T.RING].arrive()
            if it[1] in (s, 2):
                yield lambda: q_full[s].passed(n_q)
                ups[s].write(n_q, 1)
                q_ready[s].arrive()
                n_q += 1
            k += 1

    def product_warp():
        todo, n_q, unit, tile, k = deque(), [0, 0], [0, 0], 0, 0
        queries = q_ready if turn else q_full

        def ready(w):
            return p_full[w[0]][w[1] % 3].passed(w[1] // 3)

        def values():
            w = todo[0]
            yield lambda: ready(w)
            yield lambda: kv_full[w[2] % ns].passed(w[2] // ns)
            todo.popleft()
            tensor.append([pv_done[w[0]][w[1] % 3]] + ([kv_empty[w[2] % ns]] if w[3] else []))

        def until(cond, look):
            while not cond():
                yield lambda: cond() or (look and todo and ready(todo[0]))
                if look and todo and not cond() and ready(todo[0]):
                    yield from values()

        def scores(s, u, nu, last):
            if u == 0:
                yield from until(lambda: queries[s].passed(n_q[s]), looks)
                n_q[s] += 1
            n = unit[s]
            unit[s] += 1
            tensor.append([s_full[s][n % 3]] + ([kv_empty[2 * tile % ns]] if last else []) + ([q_empty[s]] if u == nu - 1 else []))
            todo.append((s, n, 2 * tile + 1, last))
            assert len(todo) <= kbuf

        while True:
            yield lambda: full[k % T.RING].passed(k // T.RING)
            it = ring[k % T.RING]
            if it is None:
                break
            empty[k % T.RING].arrive()
            nu, slot = it
            for u in range(nu):
                key = kv_full[2 * tile % ns], 2 * tile // ns
                for s in ((0, 1) if slot == 2 else (slot,)):
                    if len(todo) == kbuf:
                        yield from values()
                    if slot == 2 and s == 0:
                        yield lambda: key[0].passed(key[1])
                    elif slot != 2:
                        yield from until(lambda: key[0].passed(key[1]), True)
                    yield from scores(s, u, nu, slot != 2 or s == 1)
                tile += 1
            k += 1
        while todo:
            yield from values()

    def softmax(s):
        k = n_unit = n = n_items = 0
        while True:
            yield lambda: full[k % T.RING].passed(k // T.RING)
            it = ring[k % T.RING]
            if it is None:
                return
            nu, slot = it
            if slot in (s, 2):
                for u in range(nu):
                    yield lambda: s_full[s][n % 3].passed(n // 3)
                    if turn and u == 0:
                        ups[s].read(n_items)
                        n_items += 1
                    if u and rng.random() < 0.5:   # O is rescaled
                        yield lambda: pv_done[s][(n - 1) % 3].passed((n - 1) // 3)
                    yield None
                    scales.read(n_unit)
                    p_full[s][n % 3].arrive()
                    n, n_unit = n + 1, n_unit + 1
                yield lambda: pv_done[s][(n - 1) % 3].passed((n - 1) // 3)
            else:
                n_unit += nu
            empty[k % T.RING].arrive()
            k += 1

    each = [item_warp(), product_warp(), softmax(0), softmax(1)] + [code_warp(w) for w in range(WARPS)] + \
        ([turn_warp(0), turn_warp(1)] if turn else [])
    roles = {r: (r, None) for r in each}
    slow = rng.choice(each) if rng.random() < 0.5 else None   # one of the roles far behind the others
    while roles:
        moves = [r for r, (_, cond) in roles.items() if cond is None or cond()]
        if len(moves) > 1 and slow in moves and rng.random() < 0.95:
            moves.remove(slow)
        if copies:
            moves.append("copy")
        if tensor:
            moves.append("tensor")
        if not moves:
            raise T.Stall()
        m = rng.choice(moves)
        if m == "copy":
            copies.pop(rng.randrange(len(copies))).arrive()
        elif m == "tensor":
            for b in tensor.popleft():
                b.arrive()
        else:
            try:
                roles[m] = (m, next(m))
            except StopIteration:
                del roles[m]


def stalls(ctas, D, seed, most=8, looks=None):
    looks = looks_at_products_while_queries_come() if looks is None else looks
    rng, bad = random.Random(seed), 0
    for items in list(dict.fromkeys(tuple(i for i in c if i[0]) for c in ctas))[:most]:
        for turn in (False, True):
            try:
                run(items, D, rng, turn, looks)
            except T.Stall:
                bad += 1
    return bad


@pytest.mark.parametrize("requests,kw", [
    ([(2000, 33)] * 60, {}), ([(4096, 2048)], {}), ([(4096, 2048)], {"window": 700}), ([(1500, 800), (900, 40), (77, 77), (50, 50)], {}),
    ([(640, 300)] * 5 + [(200, 20)] * 100, {"causal": False}), ([(50000, 64)] * 2, {}), ([(100, 17)] * 2000, {}), ([(128, 128)] * 200, {})])
@pytest.mark.parametrize("heads,group", [(8, 4), (1, 1), (2, 7), (1, 128)])
@pytest.mark.parametrize("D", [64, 128])
def test_batches_do_not_stall(requests, kw, heads, group, D):
    assert stalls(T.items_of(requests, heads, group, **kw), D, seed=D, most=3) == 0


@pytest.mark.parametrize("D", [64, 128])
def test_random_lists_of_items_do_not_stall(D):
    rng = random.Random(D)
    for trial in range(200):
        items = [(rng.choice((1, 1, 1, 2, 3, 9)), rng.random() < 0.4) for _ in range(rng.randint(1, 24))]
        assert stalls([items], D, trial) == 0, items


@pytest.mark.parametrize("D", [64, 128])
def test_a_ring_too_short_is_found(D, monkeypatch):
    """The model sees places that are taken again too early."""
    monkeypatch.setitem(SCALES, D, 2)
    with pytest.raises(AssertionError, match="taken again"):
        for trial in range(200):
            stalls([[(9, False), (9, False)]], D, trial)
