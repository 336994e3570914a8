"""The order of waits in the attention kernel's ring of key and value tiles, as a model on the CPU.

A wait on an mbarrier names a phase by its last bit alone: it also passes when the phase before has not ended yet.  So whoever waits for a
turn of a ring stage must already know that the turn before it is over.  The model has the barriers (counts, bytes under way, phases), the roles
and their waits in the order of ``csrc/vt_attn.cu``; copies land in any order, products end in the order of each issuer.  Roles run under random
schedules, some of them much slower than others, and every wait that passes is compared with the phase it meant; every product with the tile
that its stage holds.  Planners and their messages are left out: roles know their pieces, which allows more schedules, not fewer."""
import random

import pytest


class Early(AssertionError):
    pass


class Barrier:
    def __init__(self, count):
        self.count, self.pending, self.bytes, self.phase = count, count, 0, 0

    def arrive(self, n=1, expect=0):
        self.bytes += expect
        self.pending -= n
        assert self.pending >= 0, "more arrivals than a phase has"
        self._turn()

    def landed(self, n=1):
        self.bytes -= n
        self._turn()

    def _turn(self):
        if self.pending == 0 and self.bytes == 0:
            self.phase += 1
            self.pending = self.count

    def passes(self, phase):                     # a wait that means `phase`, by its parity
        return (self.phase & 1) != (phase & 1)


class Ring:
    """One CTA.  pieces: (tiles, two row tiles) of each item; few: an issuer per stream.

    Planted mistakes: clean_first, the few-rows issuer waits for the values before it waits for the weights; blind, the producers ask for a stage
    without having seen that the other one's tile in it was loaded."""

    def __init__(self, pieces, stages, few, rng, clean_first=False, blind=False):
        self.pieces, self.ST, self.few, self.rng = pieces, stages, few, rng
        self.clean_first, self.blind = clean_first, blind
        self.full, self.empty = [Barrier(1) for _ in range(stages)], [Barrier(3) for _ in range(stages)]
        self.clean = [Barrier(1) for _ in range(stages)]
        self.q_full, self.q_empty = [Barrier(1) for _ in range(2)], [Barrier(3 if few else 1) for _ in range(2)]
        self.s_full, self.p_full = [Barrier(1) for _ in range(2)], [Barrier(1) for _ in range(2)]
        self.o_full, self.meet = Barrier(2 if few else 1), Barrier(2)
        self.holds = [None] * stages             # the place whose tile lies in a stage
        self.copies, self.queues = [], {}        # under way: (barrier, stage, place); what an issuer's products and commits do, in order

    # places of K(j) and V(j) in the order of loads
    @staticmethod
    def k_at(n, j):
        return 0 if j == 0 else 2 * j - 1

    @staticmethod
    def v_at(n, j):
        return 2 * j + 2 if j + 1 < n else 2 * j + 1

    def producer(self, values):
        loads = q_n = 0
        mine = set()
        for n, dual in self.pieces:
            if not values:
                for _ in range(1 + dual):
                    if q_n >= 2:
                        yield self.q_empty[q_n & 1], q_n // 2 - 1
                    self.q_full[q_n & 1].arrive(expect=1)
                    self.copies.append((self.q_full[q_n & 1], None, None))
                    q_n += 1
            for j in range(n):
                place = loads + (self.v_at if values else self.k_at)(n, j)
                turn, st = divmod(place, self.ST)
                if turn > 0:
                    if not self.blind and place - self.ST not in mine:
                        yield self.clean[st], turn - 1
                    yield self.empty[st], turn - 1
                mine.add(place)
                self.full[st].arrive(expect=1)
                self.copies.append((self.full[st], st, place))
            loads += 2 * n

    def cleaner(self):
        loads = 0
        for n, dual in self.pieces:
            for place in range(loads, loads + 2 * n):
                turn, st = divmod(place, self.ST)
                yield self.full[st], turn
                self.reads(place)
                yield None                       # takes a while
                self.reads(place)
                self.clean[st].arrive()
                self.empty[st].arrive(1 if dual else 2)
            loads += 2 * n

    def reads(self, place):
        if self.holds[place % self.ST] != place:
            raise Early(f"place {place}: the stage holds {self.holds[place % self.ST]}")

    def issuer(self, name, own):
        queue = self.queues[name] = []
        product = lambda place: queue.append(lambda: self.reads(place))          # noqa: E731
        commit = lambda bar: queue.append(bar.arrive)                            # noqa: E731
        loads = q_n = item = 0
        p_phase = [0, 0]
        for n, dual in self.pieces:
            H = n << dual
            if self.few:
                yield self.q_full[q_n & 1], q_n >> 1
            for i in range(own - 2, H, 2 if self.few else 1):
                s = i & 1
                more = i + 2 < H
                if i >= 0:
                    place = loads + self.v_at(n, i >> dual)
                    turn, st = divmod(place, self.ST)
                    waits = [(self.clean[st], turn), (self.p_full[s], p_phase[s])]
                    if self.few and i < 2 and self.ST < 7 and not self.clean_first:
                        waits.reverse()
                    yield waits[0]
                    keys = False                 # the next keys are there already
                    if not self.few and more and i + 2 > dual:
                        ahead = loads + self.k_at(n, (i + 2) >> dual)
                        keys = self.full[ahead % self.ST].passes(ahead // self.ST)
                        if keys and self.full[ahead % self.ST].phase != ahead // self.ST + 1:
                            raise Early(f"{name}: place {ahead} looks loaded")
                    yield waits[1]
                    p_phase[s] += 1
                    product(place)
                    commit(self.empty[st])
                    if not self.few and i == H - 1:
                        commit(self.o_full)
                if more:
                    place = loads + self.k_at(n, (i + 2) >> dual)
                    turn, st = divmod(place, self.ST)
                    qn = q_n + (s if dual else 0)
                    if not self.few and i + 2 <= dual:
                        yield self.q_full[qn & 1], qn >> 1
                    if i < 0 or not keys:
                        yield self.full[st], turn
                    product(place)
                    commit(self.s_full[s])
                    commit(self.empty[st])
                    if not self.few and (i + 2) >> dual == n - 1:
                        commit(self.q_empty[qn & 1])
            if self.few:
                if item > 0:
                    yield self.o_full, item - 1
                item += 1
                commit(self.q_empty[q_n & 1])
                commit(self.o_full)
            loads += 2 * n
            q_n += 1 + dual

    def softmax(self, s):
        s_phase = meets = item = 0
        for n, dual in self.pieces:
            for _ in range(s, n << dual, 2):
                yield self.s_full[s], s_phase
                s_phase += 1
                yield None
                self.p_full[s].arrive()
            yield self.o_full, item
            for last in (False, True):
                self.meet.arrive()
                yield self.meet, meets
                meets += 1
            if self.few and s == 0:
                self.q_empty[item & 1].arrive()
            item += 1

    def run(self):
        rng = self.rng
        roles = {"k": self.producer(False), "v": self.producer(True), "clean": self.cleaner(), "s0": self.softmax(0), "s1": self.softmax(1),
                 "i0": self.issuer("i0", 0)}
        if self.few:
            roles["i1"] = self.issuer("i1", 1)
        waiting = {name: None for name in roles}
        weight = lambda: 10.0 ** rng.uniform(-3, 0)                              # noqa: E731
        speed = {name: weight() for name in list(roles) + ["copy", "q0", "q1"]}
        while True:
            ready = [name for name in roles if waiting[name] is None or waiting[name][0].passes(waiting[name][1])]
            ready += ["copy"] * bool(self.copies) + [q for q, i in (("q0", "i0"), ("q1", "i1")) if self.queues.get(i)]
            if not ready:
                assert not roles, f"{sorted(roles)} wait for ever"
                return
            if rng.random() < 0.02:
                speed[rng.choice(list(speed))] = weight()
            name = rng.choices(ready, [speed[r] for r in ready])[0]
            if name == "copy":
                bar, st, place = self.copies.pop(rng.randrange(len(self.copies)))
                if st is not None:
                    self.holds[st] = place
                bar.landed()
            elif name in ("q0", "q1"):
                self.queues["i" + name[1]].pop(0)()
            else:
                if waiting[name] is not None and waiting[name][0].phase != waiting[name][1] + 1:
                    raise Early(f"{name}: a wait for phase {waiting[name][1]} passed at phase {waiting[name][0].phase}")
                try:
                    waiting[name] = next(roles[name])
                except StopIteration:
                    del roles[name]


def schedules(seed, count, stages, few, **mistakes):
    rng = random.Random(seed)
    for _ in range(count):
        pieces = [(rng.choice((1, 1, 2, 3, 3, 4, 5, 6, 9)), 0 if few else rng.randint(0, 1)) for _ in range(rng.randint(2, 7))]
        Ring(pieces, stages, few, rng, **mistakes).run()


# few rows: 5 stages with heads of 128, 12 with heads of 64; more rows: 5 or 6, 12
@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("stages", [5, 6, 7, 8, 9, 11, 12])
def test_no_wait_passes_a_phase_early(stages, few):
    schedules(100 * stages + few, 250, stages, few)


def test_all_short_sequences_of_pieces_at_five_stages():
    rng = random.Random(7)
    for a in range(1, 7):
        for b in range(1, 7):
            for c in range(1, 4):
                for _ in range(3):
                    Ring([(a, 0), (b, 0), (c, 0), (4, 0)], 5, True, rng).run()


@pytest.mark.parametrize("mistake", ["clean_first", "blind"])
def test_the_model_sees_a_wait_out_of_order(mistake):
    with pytest.raises(Early):
        schedules(1, 2000, 5, True, **{mistake: True})
