"""The waits of the shared-prefix attention kernel (csrc/prefix_attn.cu: one producer, an issuer and a softmax team per tile,
a ring of eight K / V slots), walked on the CPU under loads and products that complete in any order.

The model keeps the kernel's barriers and the order in which each role waits and arrives; a team's four warps are one role.
A barrier's wait asks for a parity, as on the device, so it returns early when the barrier is two phases behind.  The walk
fails where a role waits so, where a product or a clear meets a slot that holds anything but its block, where a slot or
an accumulator is overwritten while it is needed, and where nobody can go on.
"""
import random

import pytest

SLOTS = 8


class Broken(Exception):
    pass


class Bar:
    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self, n=1):
        for _ in range(n):
            self.left -= 1
            if self.left == 0:
                self.done, self.left = self.done + 1, self.count

    def over(self, parity):
        return self.done % 2 != parity


class Walk:
    """items: (dual, blocks, ends inside a page).  v_first: an item's first P V waits for its V before the epilogues of the item
    before are over, as the kernel once did."""

    def __init__(self, items, seed, v_first=False):
        self.items, self.rng, self.v_first = items, random.Random(seed), v_first
        self.kv_full, self.kv_empty = [Bar(1) for _ in range(SLOTS)], [Bar(2) for _ in range(SLOTS)]
        self.q_full, self.q_free, self.o_free, self.x_ready = Bar(1), Bar(2), Bar(2), Bar(2)
        self.s_full, self.p_full = [[Bar(1), Bar(1)] for _ in "01"], [[Bar(1), Bar(1)] for _ in "01"]
        self.pv_done, self.o_full = [Bar(1), Bar(1)], [Bar(1), Bar(1)]
        self.slot = [None] * SLOTS                 # what has landed
        self.q = None
        self.o = [None, None]                      # (item, blocks summed) of a team's accumulator
        self.o_needed = [set(), set()]             # teams whose epilogue has yet to read it
        self.loads, self.mma = [], [[], []]        # under way: loads in any order, a team's products in order

    def wait(self, bar, n):
        """Waits for the bar's phase n (counted from 0), by its parity."""
        if bar.done < n:
            raise Broken("a wait two phases ahead")
        while not bar.over(n % 2):
            yield
        if bar.done < n + 1:
            raise Broken("a wait returned early")

    def blind_wait(self, bar, n):
        """The same without the look behind the parity."""
        while not bar.over(n % 2):
            yield

    def blocks(self, i, team):
        dual, n, _ = self.items[i]
        return range(n) if dual else range(team, n, 2)

    def producer(self):
        pos = 0
        for i, (dual, n, _) in enumerate(self.items):
            for b in range(n):
                for kv in "KV":
                    slot, use = pos % SLOTS, pos // SLOTS
                    if use:
                        yield from self.wait(self.kv_empty[slot], use - 1)
                    self.slot[slot] = None
                    self.loads.append((slot, (i, b, kv)))
                    pos += 1
                    if kv == "K" and b == 0:
                        if i:
                            yield from self.wait(self.q_free, i - 1)
                        self.q = None
                        self.loads.append((None, i))
                    yield

    def issuer(self, team):
        base, n_qk, n_pv = 0, 0, 0
        put = self.mma[team].append
        wait_v = self.blind_wait if self.v_first else self.wait
        for i, (dual, n, _) in enumerate(self.items):
            mine = self.blocks(i, team)
            yield from self.wait(self.q_full, i)
            k_pos = lambda b: base + 2 * b

            def qk(s):
                nonlocal n_qk
                put(("qk", i, mine[s], k_pos(mine[s]) % SLOTS))
                put(("commit", self.s_full[team][n_qk % 2]))
                if s == len(mine) - 1:
                    put(("commit", self.q_free))
                n_qk += 1

            for s in range(min(2, len(mine))):
                yield from self.wait(self.kv_full[k_pos(mine[s]) % SLOTS], k_pos(mine[s]) // SLOTS)
                qk(s)
            if i and not self.v_first:
                yield from self.wait(self.o_free, i - 1)
            for s in range(len(mine)):
                v = k_pos(mine[s]) + 1
                yield from wait_v(self.kv_full[v % SLOTS], v // SLOTS)
                yield from self.wait(self.p_full[team][n_pv % 2], n_pv // 2)
                if i and s == 0 and self.v_first:
                    yield from self.wait(self.o_free, i - 1)
                put(("pv", i, mine[s], v % SLOTS, team, s))
                put(("commit", self.pv_done[team]))
                yield from self.wait(self.pv_done[team], n_pv)
                self.kv_empty[v % SLOTS].arrive(1 if dual else 2)
                n_pv += 1
                if s + 2 < len(mine):
                    k = k_pos(mine[s + 2])
                    yield from self.wait(self.kv_full[k % SLOTS], k // SLOTS)
                    qk(s + 2)
            if not len(mine):
                put(("commit", self.q_free))
                if i and self.v_first:
                    yield from self.wait(self.o_free, i - 1)
            put(("commit", self.o_full[team]))
            base += 2 * n

    def softmax(self, team):
        base, step = 0, 0
        for i, (dual, n, partial) in enumerate(self.items):
            mine = self.blocks(i, team)
            for s, b in enumerate(mine):
                pos = base + 2 * b
                yield from self.wait(self.s_full[team][step % 2], step // 2)
                self.kv_empty[pos % SLOTS].arrive(1 if dual else 2)
                if partial and b == n - 1:
                    v = pos + 1
                    yield from self.wait(self.kv_full[v % SLOTS], v // SLOTS)
                    if self.slot[v % SLOTS] != (i, b, "V"):
                        raise Broken("rows of another block are cleared")
                if s and self.rng.random() < 0.5:                      # the maximum moves: O is rescaled
                    yield from self.wait(self.pv_done[team], step - 1)
                self.p_full[team][step % 2].arrive()
                step += 1
                yield
            yield from self.wait(self.o_full[team], i)
            if not dual:
                yield from self.wait(self.o_full[team ^ 1], i)
                self.x_ready.arrive()
                yield from self.wait(self.x_ready, sum(not d for d, _, _ in self.items[:i]))
            for t in [team] if dual else [0, 1]:
                if len(self.blocks(i, t)) and self.o[t] != (i, len(self.blocks(i, t))):
                    raise Broken("an accumulator that is not the item's")
                self.o_needed[t].discard(team)
            self.o_free.arrive()
            base += 2 * n
            yield

    def advance_mma(self, team):
        what, *a = self.mma[team].pop(0)
        if what == "commit":
            a[0].arrive()
        elif what == "qk":
            i, b, slot = a
            if self.slot[slot] != (i, b, "K") or self.q != i:
                raise Broken("Q K^T of another block")
        else:
            i, b, slot, t, s = a
            if self.slot[slot] != (i, b, "V"):
                raise Broken("P V of another block")
            if s == 0:
                if self.o_needed[t]:
                    raise Broken("an accumulator is overwritten before it was read")
                self.o_needed[t] = {t} if self.items[i][0] else {0, 1}
                self.o[t] = (i, 0)
            self.o[t] = (i, self.o[t][1] + 1)

    def land(self, k):
        slot, what = self.loads.pop(k)
        if slot is None:
            self.q = what
            self.q_full.arrive()
        else:
            self.slot[slot] = what
            self.kv_full[slot].arrive()

    def run(self):
        rng = self.rng
        roles = [self.producer(), self.issuer(0), self.issuer(1), self.softmax(0), self.softmax(1)]
        slow = rng.choice([1.0, 0.1, 0.01])                            # how soon a V lands beside everything else
        idle = 0
        while roles or self.mma[0] or self.mma[1] or self.loads:
            before = self.state(roles)
            x = rng.random()
            if x < 0.25 and self.loads:
                k = rng.randrange(len(self.loads))
                if self.loads[k][0] is None or self.loads[k][1][2] == "K" or rng.random() < slow or idle > 300:
                    self.land(k)
            elif x < 0.5:
                t = rng.randrange(2)
                if self.mma[t]:
                    self.advance_mma(t)
            elif roles:
                r = rng.choice(roles)
                try:
                    next(r)
                except StopIteration:
                    roles.remove(r)
            idle = idle + 1 if self.state(roles) == before else 0
            if idle > 5000:
                raise Broken("nobody can go on")

    def state(self, roles):
        bars = [*self.kv_full, *self.kv_empty, self.q_full, self.q_free, self.o_free, self.x_ready, *self.pv_done, *self.o_full,
                *(b for t in (*self.s_full, *self.p_full) for b in t)]
        return [(b.done, b.left) for b in bars], len(roles), len(self.loads), [len(m) for m in self.mma]


def random_items(rng):
    return [(rng.random() < 0.4, rng.choice([1, 1, 2, 3, 3, 4, 5, 7, 9]), rng.random() < 0.5) for _ in range(rng.randint(2, 7))]


@pytest.mark.parametrize("part", range(4))
def test_every_wait_and_every_slot(part):
    for seed in range(150 * part, 150 * (part + 1)):
        Walk(random_items(random.Random(seed)), seed).run()


@pytest.mark.parametrize("items", [[(False, 3, True), (False, 3, True)], [(False, 3, False), (True, 1, True)], [(False, 1, True)] * 6,
                                   [(True, 1, True), (False, 1, True), (False, 2, True)], [(False, 5, True), (True, 5, True), (False, 4, True)]])
def test_odd_singles_before_other_items(items):
    for seed in range(100):
        Walk(items, seed).run()


def test_the_walk_sees_a_wait_for_v_before_the_item_before_is_over():
    with pytest.raises(Broken, match="another block|early"):
        for seed in range(300):
            Walk([(False, 3, False), (False, 3, False), (False, 3, False)], seed, v_first=True).run()
