"""The barriers of the tile kernel of cached attention (csrc/attention_cached_tc.cuh, attn_tiles_kernel) under random schedules.

A model of the roles (producer, an MMA issuer per row tile, the warp that looks the values over, two groups of four softmax warps), in
which copies end in any order, products in order, and a role can be held up at any point.  mbarriers are modelled as they are: a wait
names a parity, so a role that is overtaken by two phases cannot tell.  Who gives a ring place free is taken from the source."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_24273_b200", "csrc", "attention_cached_tc.cuh")


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.bytes = self.phase = 0

    def _check(self):
        if self.pending == 0 and self.bytes == 0:
            self.phase, self.pending = self.phase + 1, self.count

    def arrive(self, expect=0):
        assert self.pending > 0, "more arrivals than the barrier counts"
        self.pending -= 1
        self.bytes += expect
        self._check()

    def land(self):
        self.bytes -= 1
        self._check()

    def passed(self, parity):
        return self.phase & 1 != parity


def simulate(seed, ring, leaves, looker_leaves, items, held):
    """items: (units, 64-slot steps, row tiles).  Returns None, or what every role waits for when none can go on."""
    rnd = random.Random(seed)
    bars = {(n, i): Barrier(c) for n, c in (("kv_full", 1), ("kv_empty", leaves), ("v_ready", 1)) for i in range(ring)}
    bars |= {(n, i): Barrier(c) for n, c in (("s_full", 1), ("p_full", 4), ("o_done", 1)) for i in range(4)}
    bars |= {("q_full", 0): Barrier(1), ("q_empty", 0): Barrier(2)}
    copies, pipes, place, looked = [], ([], []), [None] * ring, set()

    def producer():
        e = n = 0
        for units, _, _ in items:
            for u in range(units):
                for kv in range(2):
                    at = e % ring
                    yield "kv_empty", at, (e // ring) & 1 ^ 1
                    place[at] = None
                    bars["kv_full", at].arrive(1)

                    def landed(at=at, e=e):
                        place[at] = e
                        bars["kv_full", at].land()

                    copies.append(landed)
                    e += 1
                    yield
                    if u == 0 and kv == 0:
                        yield "q_empty", 0, n & 1 ^ 1
                        bars["q_full", 0].arrive(1)
                        copies.append(bars["q_full", 0].land)
                        n += 1
                        yield

    def issuer(x):
        e = n = p_par = 0
        commit = lambda *bar: pipes[x].append(("commit", bar, None))  # noqa: E731
        scores = lambda t, b: pipes[x].append(("product", ("s_full", 2 * x + b), t))  # noqa: E731
        for units, steps, tiles in items:
            yield "q_full", 0, n & 1
            n += 1
            if x == 1 and tiles == 1:
                bars["q_empty", 0].arrive()
                yield
                for _ in range(2 * units):
                    yield "kv_full", e % ring, (e // ring) & 1
                    assert place[e % ring] == e
                    bars["kv_empty", e % ring].arrive()
                    e += 1
                    yield
                continue
            yield "kv_full", e % ring, (e // ring) & 1
            for b in range(min(steps, 2)):
                scores(e, b)
            commit("kv_empty", e % ring)
            if steps <= 2:
                commit("q_empty", 0)
            yield
            for i in range(steps):
                b, ve = i & 1, e + 2 * (i >> 1) + 1
                ke = ve + 1
                if b == 0:
                    yield "v_ready", ve % ring, (ve // (2 * ring)) & 1
                assert ve in looked
                yield "p_full", 2 * x + b, (p_par >> b) & 1
                p_par ^= 1 << b
                pipes[x].append(("product", ("o_done", 2 * x + b), ve))
                yield
                if b == 1 or i + 1 == steps:
                    commit("kv_empty", ve % ring)
                if i + 2 < steps:
                    if b == 0:
                        yield "kv_full", ke % ring, (ke // ring) & 1
                    scores(ke, b)
                    if b == 1 or i + 3 == steps:
                        commit("kv_empty", ke % ring)
                if i + 3 == steps:
                    commit("q_empty", 0)
                yield
            e += 2 * units

    def looker():
        e = 1
        for units, _, _ in items:
            for _ in range(rnd.choice(held)):
                yield
            for _ in range(units):
                yield "kv_full", (e - 1) % ring, ((e - 1) // ring) & 1
                if looker_leaves:
                    bars["kv_empty", (e - 1) % ring].arrive()
                yield "kv_full", e % ring, (e // ring) & 1
                assert place[e % ring] == e
                for _ in range(rnd.choice(held)):
                    yield
                looked.add(e)
                bars["v_ready", e % ring].arrive()
                if looker_leaves:
                    bars["kv_empty", e % ring].arrive()
                e += 2
                yield

    def softmax(x):
        s_par = o_par = 0
        for _, steps, tiles in items:
            yield
            if x == 1 and tiles == 1:
                continue
            for i in range(steps):
                b = i & 1
                yield "s_full", 2 * x + b, (s_par >> b) & 1
                s_par ^= 1 << b
                if i and rnd.random() < 0.3:  # the maximum has grown: the last product has to be there
                    yield "o_done", 2 * x + (b ^ 1), (o_par >> (b ^ 1)) & 1 ^ 1
                bars["p_full", 2 * x + b].arrive()
                o_par ^= 1 << b
                yield
            b = steps - 1 & 1
            yield "o_done", 2 * x + b, (o_par >> b) & 1 ^ 1

    roles = {"producer": producer(), "issuer 0": issuer(0), "issuer 1": issuer(1), "looker": looker()}
    roles |= {f"softmax {x}.{k}": softmax(x) for x in range(2) for k in range(4)}
    waits = dict.fromkeys(roles)
    weight = {r: rnd.choice([1, 1, 1, 8, 40]) for r in roles}
    while roles:
        able = [r for r in roles if waits[r] is None or bars[waits[r][:2]].passed(waits[r][2])]
        events = able + [("copy", i) for i in range(len(copies))] + [("pipe", x) for x in range(2) if pipes[x]]
        if not events:
            return {r: waits[r] for r in roles}
        what = rnd.choices(events, [weight.get(v, 3) if isinstance(v, str) else 3 for v in events])[0]
        if isinstance(what, str):
            waits[what] = None
            try:
                waits[what] = next(roles[what])
            except StopIteration:
                del roles[what]
        elif what[0] == "copy":
            copies.pop(what[1])()
        else:
            kind, bar, tile = pipes[what[1]].pop(0)
            assert kind == "commit" or place[tile % ring] == tile, "a product read a place that another tile had taken"
            bars[bar].arrive()
    return None


def protocol():
    with open(SOURCE) as f:
        text = f.read()
    kernel = text[text.index("attn_tiles_kernel(const") : text.index("attn_tiles_join_kernel(const")]
    ring = int(re.search(r"AT_RING = (\d+);", text).group(1))
    leaves = int(re.search(r"mbar_init\(base \+ M::KV_EMPTY \+ 8 \* i, (\d+)\)", kernel).group(1))
    looker = kernel[kernel.index("values of masked units") : kernel.index("softmax, one row per thread")]
    return ring, leaves, len(re.findall(r"mbar_arrive\(base \+ M::KV_EMPTY", looker)) == 2


def items(rnd, one_tile):
    out = []
    for _ in range(rnd.randint(1, 12)):
        units = rnd.randint(1, 9)
        out.append((units, 2 * units - rnd.randint(0, 1), 1 if one_tile else rnd.randint(1, 2)))
    return out


@pytest.mark.parametrize("one_tile", [True, False])
@pytest.mark.parametrize("held", [[0], [0, 3], [0, 30], [0, 0, 0, 200]])
def test_every_role_ends(one_tile, held):
    ring, leaves, looker_leaves = protocol()
    for seed in range(60):
        stuck = simulate(seed, ring, leaves, looker_leaves, items(random.Random(seed + 7000), one_tile), held)
        assert stuck is None, (seed, stuck)


def test_the_model_finds_a_warp_that_is_overtaken():
    """With leave from the issuers alone, the warp that looks the values over can miss a round of its barrier."""
    found = [simulate(seed, 5, 2, False, items(random.Random(seed + 7000), True), [0, 30]) for seed in range(60)]
    assert any(f is not None and f["looker"][0] == "kv_full" for f in found)
