"""The hand-overs inside chunk_kernel, on the CPU: what no run can show, because it depends on timing."""
import os
import random
import re

import pytest

SOURCE = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_18139_b200", "csrc",
                           "chunk_kernel.cu")).read()


def test_tensor_memory_that_another_warpgroup_reads_is_fenced_on_both_sides():
    """Stream 0 reads stream 1's output block once merge_full has told it so: an mbarrier orders tensor memory only between a fence in front
    of the arrival and one behind the wait."""
    role = SOURCE[SOURCE.index("void softmax_rows"):SOURCE.index("chunk_kernel(const __grid_constant__")]
    arrival = role.index("mbar_arrive(ptx::smem_u32(&sh.merge_full))")
    wait = role.index("warp_wait(&sh.merge_full")
    reads = role.index("tmem_ld_32x16(to + kHeadDim")
    stores = [m.start() for m in re.finditer(r"tmem_(st|ld)_32x\d+\(t", role) if m.start() < arrival]
    assert max(stores) < role.rindex("tc_fence_before_sync()", 0, arrival)
    assert wait < role.index("tc_fence_after_sync()", wait) < reads
    assert role.rindex("tc_fence_before_sync()", 0, arrival) > role.index("if (!it.pair && g == 1)")


# ---- a model of the roles -------------------------------------------------------------------------------
# Roles are generators that yield what they wait for: (barrier, parity).  A scheduler lets any role go on whose wait is over, and lets copies
# land in any order; a role that it seldom picks lags behind as far as the barriers allow.
TILE = 128


def constant(name):
    return int(re.search(r"constexpr int (?:k\w+ = [^;]*, )?%s = (\d+)" % name, SOURCE).group(1))


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.phase = 0

    def arrive(self):
        assert self.pending > 0
        self.pending -= 1
        if self.pending == 0:
            self.pending, self.phase = self.count, self.phase ^ 1

    def done(self, parity):
        return self.phase != parity


class Item:
    """`pair` of query tiles, tiles of cached rows in all and of stream 0, and how many of the first tiles every row sees whole."""

    def __init__(self, pair, nt, nt0=None, seen_by_all=0):
        self.pair, self.nt, self.seen_by_all = pair, nt, seen_by_all
        self.nt0 = (nt if nt0 is None else nt0) if pair else (nt + 1) >> 1
        self.nt1 = nt if pair else nt >> 1

    def masked(self, t):
        return t >= self.seen_by_all

    def ring(self):
        """Its tiles in the order in which they come through the ring."""
        ahead = 1 if self.pair else 2
        tiles = [("K", t) for t in range(min(ahead, self.nt))]
        for t in range(self.nt):
            tiles += [("V", t)] + ([("K", t + ahead)] if t + ahead < self.nt else [])
        return tiles


class Model:
    def __init__(self, items, loaders):
        ring, self.n_flags = constant("kRing"), constant("kFlags")
        self.items, self.loaders, self.n_ring = items, loaders, ring
        one = lambda count, n: [Barrier(count) for _ in range(n)]
        self.q_full, self.q_empty, self.s_full, self.pv_done, self.o_free = one(1, 2), one(1, 2), one(1, 2), one(1, 2), one(4, 2)
        self.p_part = [one(4, 2), one(4, 2)]
        self.full, self.empty, self.dirty = one(2 + 2, ring), one(1, ring), one(1 + 2, ring)         # (and the bytes of both loaders' parts)
        self.merge_full, self.merge_free = Barrier(4), Barrier(4)
        self.tiles, self.queries, self.probabilities = [{} for _ in range(ring)], [None] * 2, [[None] * 4, [None] * 4]
        self.flags, self.copies = [0] * self.n_flags, []
        self.cleaned = {}                        # cleaning warps that are through with (item, V tile)

    def load(self, part):
        n = nq = 0
        for i, it in enumerate(self.items):
            for g in range(2 if it.pair else 1) if part == 0 else ():
                s = nq & 1
                yield self.q_empty[s], (nq >> 1 & 1) ^ 1

                def query(s=s, what=(i, g)):
                    self.queries[s] = what
                    self.q_full[s].arrive()
                self.copies.append(query)
                nq += 1
            for kind, t in it.ring():
                s, raw = n % self.n_ring, kind == "V" and it.masked(t)
                yield self.empty[s], (n // self.n_ring & 1) ^ 1
                bar = (self.dirty if raw else self.full)[s]
                if part == 0:
                    bar.arrive()
                    if not raw:
                        bar.arrive()

                def tile(s=s, bar=bar, what=(i, kind, t, raw)):
                    self.tiles[s][part] = what
                    for _ in range(2 // self.loaders):
                        bar.arrive()
                self.copies.append(tile)
                n += 1

    def has(self, s, what):
        return all(self.tiles[s].get(part) == what for part in range(self.loaders))

    def issue(self):
        n = nq = 0
        p_parity, o_parity = [0, 0], [1, 1]

        def qk(g, s, t):
            assert self.has(s, (i, "K", t, False))
            assert self.queries[nq + (g if it.pair else 0) & 1] == (i, g if it.pair else 0)
            self.s_full[g].arrive()

        def pv(g, s, t):
            for half in range(2):
                yield self.p_part[g][half], p_parity[g]
            p_parity[g] ^= 1
            assert self.has(s, (i, "V", t, False)) and self.probabilities[g] == [(i, t)] * 4
            self.pv_done[g].arrive()

        for i, it in enumerate(self.items):
            sets, ahead = (2, 1) if it.pair else (1, 2)
            for g in range(sets):
                yield self.q_full[nq + g & 1], nq + g >> 1 & 1
            streams = lambda t: [g for g in ((0, 1) if it.pair else (t & 1,)) if t < (it.nt0, it.nt)[g] or not it.pair]
            for t in range(min(ahead, it.nt)):
                yield self.full[n % self.n_ring], n // self.n_ring & 1
                for g in streams(t):
                    qk(g, n % self.n_ring, t)
                self.empty[n % self.n_ring].arrive()
                n += 1
            queries_left = it.nt > ahead
            if not queries_left:
                for g in range(sets):
                    self.q_empty[nq + g & 1].arrive()
            for g in range(2):
                if (it.nt0, it.nt1)[g] > 0:
                    yield self.o_free[g], o_parity[g]
                    o_parity[g] ^= 1
            for t in range(it.nt):
                v, k = n % self.n_ring, None
                yield self.full[v], n // self.n_ring & 1
                n += 1
                if t + ahead < it.nt:
                    k = n % self.n_ring
                    yield self.full[k], n // self.n_ring & 1
                    n += 1
                for g in streams(t):
                    yield from pv(g, v, t)
                    if k is not None and g in streams(t + ahead) and not (it.pair and g == 1):
                        qk(g, k, t + ahead)
                self.empty[v].arrive()
                if k is not None:
                    if it.pair:
                        qk(1, k, t + ahead)
                    self.empty[k].arrive()
                    if t + ahead + 1 == it.nt:
                        for g in range(sets):
                            self.q_empty[nq + g & 1].arrive()
            nq += sets

    def clean(self, warp):
        n, parity = 0, [0] * self.n_ring
        for i, it in enumerate(self.items):
            for t in range(it.nt):
                if not it.masked(t):
                    continue
                s = (n + it.ring().index(("V", t))) % self.n_ring
                yield self.dirty[s], parity[s]
                parity[s] ^= 1
                assert all(self.tiles[s][part][:3] == (i, "V", t) for part in range(self.loaders))
                self.flags[i % self.n_flags] = i + 1
                self.cleaned[i, t] = self.cleaned.get((i, t), 0) + 1
                for part in range(self.loaders) if self.loaders == 2 or self.cleaned[i, t] == 2 else ():
                    self.tiles[s][part] = (i, "V", t, False)
                for _ in range(4 if self.loaders == 2 else 2):
                    self.full[s].arrive()
            n += 2 * it.nt

    def softmax(self, g, warp):
        n = merges = 0
        for i, it in enumerate(self.items):
            nt = (it.nt0, it.nt1)[g]
            for j in range(nt):
                yield self.s_full[g], n & 1
                if j > 0:
                    yield self.pv_done[g], n - 1 & 1
                self.probabilities[g][warp] = (i, j if it.pair else 2 * j + g)
                self.p_part[g][0].arrive()
                yield self.s_full[g], n & 1
                self.p_part[g][1].arrive()
                n += 1
            if nt > 0:
                yield self.pv_done[g], n - 1 & 1
            if not it.pair:
                if g == 1:
                    yield self.merge_free, (merges & 1) ^ 1
                    self.merge_full.arrive()
                    merges += 1
                    continue
                yield self.merge_full, merges & 1
                merges += 1
                self.merge_free.arrive()
            if any(it.masked(t) for t in range(nt if it.pair else it.nt)):           # (tiles that this stream's rows see)
                assert self.flags[i % self.n_flags] == i + 1, "a later item's flag lies over this one's"
            if nt > 0:
                self.o_free[g].arrive()
            if not it.pair and it.nt1 > 0:
                self.o_free[1].arrive()

    def run(self, rng, slow):
        """`slow`: how seldom a role is picked, by the beginning of its name."""
        roles = {"load0": self.load(0), "issue": self.issue(), "clean0": self.clean(0)}
        roles.update({"load1": self.load(1)} if self.loaders == 2 else {"clean1": self.clean(1)})
        roles.update({"soft%d%d" % (g, w): self.softmax(g, w) for g in range(2) for w in range(4)})
        waits = {name: next(role, None) for name, role in roles.items()}
        weight = {name: min([f for k, f in slow.items() if name.startswith(k)] + [0.05 + rng.random()]) for name in [*roles, "copy"]}
        while any(waits.values()):
            ready = [name for name, w in waits.items() if w and w[0].done(w[1])] + (["copy"] if self.copies else [])
            assert ready, "nobody can go on: %s" % [name for name, w in waits.items() if w]
            name = rng.choices(ready, [weight[x] for x in ready])[0]
            if name == "copy":
                self.copies.pop(rng.randrange(len(self.copies)))()
            else:
                waits[name] = next(roles[name], None)


def draw_items(rng):
    """Short items are the rule: they let the loads run ahead of the outputs by most items."""
    items = []
    for _ in range(rng.randint(2, 12)):
        pair, nt = rng.random() < 0.4, rng.choice([1, 1, 1, 2, 3, 6])
        seen = rng.choice([0, 0, nt - 1, nt])
        items.append(Item(pair, nt, rng.choice([nt, max(nt - 1, 0)]), max(seen, 0)))
    return items


@pytest.mark.parametrize("loaders", [1, 2])
@pytest.mark.parametrize("slow", ["", "soft0", "soft1", "soft00", "soft12", "issue", "clean", "load", "copy"])
def test_hand_overs_in_any_order(slow, loaders):
    """Every role meets the tiles, queries and probabilities that are meant for it, nobody waits for good, and what was found among an item's
    values is still to be seen when its outputs are written."""
    for seed in range(60):
        rng = random.Random(seed)
        Model(draw_items(rng), loaders).run(rng, {slow: 1e-6} if slow else {})


def test_flags_of_items_that_are_in_flight_together_lie_apart():
    """A pair of query tiles whose stream 1 is late, then single tiles of which stream 1 has nothing: the cleaning warps come as far as the
    fourth item after it."""
    for n in range(1, 8):
        for seed in range(10):
            Model([Item(True, 1, 1)] + [Item(False, 1)] * n, 1).run(random.Random(seed), {"soft1": 1e-9})
