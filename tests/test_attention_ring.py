"""The waits between the roles of the paged attention's kernel, as a model on the CPU: no order of the roles may leave all of
them waiting, and no wait for a parity may meet a barrier that is two phases away from it.

The model has the roles as the kernel has them (the warp of items and keys, that of values, that of the products, the two
slots' softmax warps, the tensor core's completions and the copies' landings), each as a generator that yields what it waits
for, run one step at a time in a random order.  Its sizes are read from the kernel's source, as is whether an item without keys
takes a place in the ring of items: the product warp issues what it holds back only for an item's units, and a ring full of
items that have none leaves all waiting.  The items come from batches by the kernel's own rule of
ranges and cuts, which is checked on the way (each unit once, parts counted alike by all), and at random."""
import os
import random
import re
from collections import deque

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2408_04323_gb300", "csrc", "paged_attn.cu")
TEXT = re.sub(r"//[^\n]*", "", open(SRC).read())
SMS = 152


def number(name):
    return int(re.search(rf"constexpr int (?:\w+ = \d+, )?{name} = (\d+)", TEXT).group(1))


RING, KEYS, ROWS = number("kRing"), number("kKeys"), number("kRows")
ITEM_COST, PAIR_COST, MIN_RANGE = number("kItemCost"), number("kPairCost"), number("kMinRange")
SNAP_MIN, SNAP_MAX = number("kSnapMin"), number("kSnapMax")
STAGES = dict(zip((128, 64), map(int, re.search(r"kStages = \(D == 128 \? (\d+) : (\d+)\)", TEXT).groups())))
BUFS = dict(zip((128, 64), map(int, re.search(r"kBuf = D == 128 \? (\d+) : (\d+)", TEXT).groups())))


def empty_items_have_a_place():
    """Whether the warp of items hands on items without keys."""
    loop = TEXT[TEXT.index("while (p < B1 && wait.ok) {"):]
    before = loop[:loop.index("items[ring] = it;")]
    return re.search(r"if \(units == 0\) \{\s*no_keys<D>\(a, it\);\s*continue;\s*\}", before) is None


# ---------------------------------------------------------------------------------------------- the ranges' items

def seen(kv, n, tok0, nt, causal, window):
    p0 = kv - n + tok0
    end = min(kv, p0 + nt) if causal else kv
    begin = max(0, p0 + 1 - window) if window else 0
    return (begin, end) if end > begin else (0, 0)


def items_of(requests, heads, group, causal=True, window=0, sms=SMS):
    """Per CTA its items as (units, pair, parts), of requests [(length, new tokens)]; checks that all units are taken once."""
    toks = ROWS // group
    per = 2 * toks
    row, at = [], 0   # of one head: (start, units, pair)
    for kv, n in requests:
        for j in range(-(-n // per)):
            nt = min(per, n - j * per)
            b, e = seen(kv, n, j * per, nt, causal, window)
            units = -(-e // KEYS) - b // KEYS
            cost = PAIR_COST if n - j * per > toks else ITEM_COST
            row.append((at, cost, units, nt > toks))
            at += cost + units
    total = at * heads
    width = max(-(-total // sms), MIN_RANGE)
    snap = max(SNAP_MIN, min(SNAP_MAX, width // 4))
    ctas = [[] for _ in range(sms)]
    for h in range(heads):
        for p, cost, units, pair in row:
            p += h * at
            s = p + cost

            def cut(b):
                return units if b >= s + units else 0 if b - s < snap else units if s + units - b < snap else b - s

            taken, parts = 0, []
            for c in range(max(0, p // width - 1), min(sms, (s + units) // width + 2)):
                B0, B1 = min(total, c * width), min(total, c * width + width)
                lo, hi = cut(B0), cut(B1)
                if not (B0 < B1 and p < B1 and (hi > lo if units else p >= B0)):
                    continue
                assert lo == taken
                taken = hi
                parts.append(c)
                first, n_parts = c, 1
                if hi - lo < units:
                    first = (s + snap - 1) // width
                    n_parts = (s + units - snap) // width - first + 1
                ctas[c].append((hi - lo, pair, (first, n_parts)))
            assert taken == units and parts and parts == list(range(parts[0], parts[0] + len(parts)))
            assert all(ctas[c][-1][2] == (parts[0], len(parts)) for c in parts)
    return [[(nu, pair) for nu, pair, _ in items] for items in ctas]


# ---------------------------------------------------------------------------------------------- the roles

class Stall(Exception):
    pass


class Barrier:
    def __init__(self, count=1):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1

    def passed(self, use):
        """A wait for the parity of use `use`: sound only within a phase of it."""
        assert use <= self.done <= use + 1, (use, self.done)
        return self.done == use + 1


def run(items, D, rng):
    """One CTA's items (units, pair) through the roles in a random order; raises Stall if all wait."""
    ns, kbuf = STAGES[D], BUFS[D]
    listed, turn = [], 0
    for nu, pair in items:
        listed.append((nu, 2 if pair else turn))
        if not pair:
            turn ^= 1
    full, empty = [Barrier() for _ in range(RING)], [Barrier(4) for _ in range(RING)]
    kv_full, kv_empty = [Barrier() for _ in range(ns)], [Barrier() for _ in range(ns)]
    q_full, q_empty = [Barrier(), Barrier()], [Barrier(), Barrier()]
    s_full, p_full, pv_done = ([[Barrier() for _ in range(3)] for _ in range(2)] for _ in range(3))
    ring = [None] * RING
    copies, tensor = [], deque()   # copies land in any order, the tensor core's work completes in its own

    def load(i):   # a tile of keys (i even) or values (i odd)
        st = i % ns
        if i >= ns:
            yield lambda: kv_empty[st].passed(i // ns - 1)
        copies.append(kv_full[st])

    def item_warp():
        at, n_q = 0, [0, 0]
        for k, it in enumerate(listed + [None]):
            if k >= RING:
                yield lambda: empty[k % RING].passed(k // RING - 1)
            ring[k % RING] = it
            full[k % RING].arrive()
            for u in range(it[0] if it else 0):
                yield from load(at)
                at += 2
                for s in (0, 1):
                    if u == 0 and it[1] in (s, 2):
                        if n_q[s]:
                            yield lambda: q_empty[s].passed(n_q[s] - 1)
                        copies.append(q_full[s])
                        n_q[s] += 1

    def value_warp():
        at, k = 1, 0
        while True:
            yield lambda: full[k % RING].passed(k // RING)
            it = ring[k % RING]
            if it is None:
                return
            empty[k % RING].arrive()
            for _ in range(it[0]):
                yield from load(at)
                at += 2
            k += 1

    def product_warp():
        todo, n_q, unit, tile, k = deque(), [0, 0], [0, 0], 0, 0

        def ready(w):
            s, n, v, _ = w
            return p_full[s][n % 3].passed(n // 3) and kv_full[v % ns].passed(v // ns)

        def values():
            w = todo[0]
            yield lambda: p_full[w[0]][w[1] % 3].passed(w[1] // 3)
            yield lambda: kv_full[w[2] % ns].passed(w[2] // ns)
            todo.popleft()
            tensor.append([pv_done[w[0]][w[1] % 3]] + ([kv_empty[w[2] % ns]] if w[3] else []))

        def scores(s, u, nu, last):
            if u == 0:
                yield lambda: q_full[s].passed(n_q[s])
                n_q[s] += 1
            n = unit[s]
            unit[s] += 1
            tensor.append([s_full[s][n % 3]] + ([kv_empty[2 * tile % ns]] if last else []) + ([q_empty[s]] if u == nu - 1 else []))
            todo.append((s, n, 2 * tile + 1, last))
            assert len(todo) <= kbuf

        while True:
            yield lambda: full[k % RING].passed(k // RING)
            it = ring[k % RING]
            if it is None:
                break
            empty[k % RING].arrive()
            nu, slot = it
            for u in range(nu):
                key = kv_full[2 * tile % ns], 2 * tile // ns
                if slot == 2:
                    for s in (0, 1):
                        if len(todo) == kbuf:
                            yield from values()
                        if s == 0:
                            yield lambda: key[0].passed(key[1])
                        yield from scores(s, u, nu, s == 1)
                else:
                    if len(todo) == kbuf:
                        yield from values()
                    while not key[0].passed(key[1]):
                        yield lambda: key[0].passed(key[1]) or (todo and ready(todo[0]))
                        if todo and ready(todo[0]):
                            yield from values()
                    yield from scores(slot, u, nu, True)
                tile += 1
            k += 1
        while todo:
            yield from values()

    def softmax(s):
        k = n_unit = n = 0
        while True:
            yield lambda: full[k % RING].passed(k // RING)
            it = ring[k % RING]
            if it is None:
                return
            nu, slot = it
            if slot in (s, 2):
                for u in range(nu):
                    yield lambda: s_full[s][n % 3].passed(n // 3)
                    if u and rng.random() < 0.5:   # O is rescaled
                        yield lambda: pv_done[s][(n - 1) % 3].passed((n - 1) // 3)
                    if rng.random() < 0.5:         # values are looked through
                        v = 2 * n_unit + 1
                        yield lambda: kv_full[v % ns].passed(v // ns)
                    p_full[s][n % 3].arrive()
                    n, n_unit = n + 1, n_unit + 1
                if nu:
                    yield lambda: pv_done[s][(n - 1) % 3].passed((n - 1) // 3)
            else:
                n_unit += nu
            empty[k % RING].arrive()
            k += 1

    roles = {r: (r, None) for r in (item_warp(), value_warp(), product_warp(), softmax(0), softmax(1))}
    while roles:
        moves = [r for r, (_, cond) in roles.items() if cond is None or cond()]
        if copies:
            moves.append("copy")
        if tensor:
            moves.append("tensor")
        if not moves:
            raise Stall()
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


def stalls(ctas, D, places, seed=0, most=12):
    """How many of the given lists stall (alike ones are run once); places: whether empty items take a place in the ring."""
    rng, bad = random.Random(seed), 0
    for items in list(dict.fromkeys(tuple(c) for c in ctas))[:most]:
        try:
            run([i for i in items if i[0] or places], D, rng)
        except Stall:
            bad += 1
    return bad


REFUSED = {   # (length, new tokens): a length of 0 is a refused request's
    "decodes and a refused prompt": ([(64 + 7 * i, 1) for i in range(249)] + [(0, 512)], 128),
    "few decodes and two refused": ([(100, 1)] * 40 + [(0, 1)] * 2, 128),
    "heads of 64, every 16th refused": ([(0 if i % 16 == 0 else 100, 1) for i in range(200)], 64),
    "served decodes, then refused ones": ([(300, 1)] * 300 + [(0, 1)] * 300, 128),
    "tokens before their sequence": ([(300, 3000)], 128),
}


@pytest.mark.parametrize("name", REFUSED)
def test_items_without_keys_do_not_stall(name):
    requests, D = REFUSED[name]
    ctas = sorted(items_of(requests, 8, 4), key=lambda c: -sum(nu == 0 for nu, _ in c))   # those that can stall first
    assert stalls(ctas, D, True) > 0   # with places for all, the batch is one that stalls
    assert stalls(ctas, D, empty_items_have_a_place()) == 0


@pytest.mark.parametrize("requests,kw", [
    ([(2000, 1)] * 60, {}), ([(4096, 2048)], {}), ([(4096, 2048)], {"window": 700}), ([(1500, 800), (900, 1), (77, 77), (5, 5)], {}),
    ([(640, 300)] * 5 + [(200, 1)] * 100, {"causal": False}), ([(50000, 1)] * 2, {}), ([(1, 1)], {}), ([(0, 1)], {}),
    ([(100, 1)] * 2000, {}), ([(128, 128)] * 200, {})])
@pytest.mark.parametrize("heads,group", [(8, 4), (1, 1), (2, 7), (1, 128)])
@pytest.mark.parametrize("D", [64, 128])
def test_batches_do_not_stall(requests, kw, heads, group, D):
    assert stalls(items_of(requests, heads, group, **kw), D, empty_items_have_a_place(), seed=D, most=4) == 0


@pytest.mark.parametrize("D", [64, 128])
def test_random_lists_of_items_do_not_stall(D):
    rng = random.Random(D)
    held = 0
    for trial in range(300):
        empty = rng.choice((0.0, 0.2, 0.6, 0.9))
        items = [(0 if rng.random() < empty else rng.choice((1, 1, 2, 3, 9)), rng.random() < 0.4) for _ in range(rng.randint(1, 24))]
        held += stalls([items], D, True, seed=trial)
        assert stalls([items], D, empty_items_have_a_place(), seed=trial) == 0, items
    assert held > 10   # with places for all, such lists do stall
