"""The barriers of the prefix attention's CTA as a model on the host: its roles as they wait and arrive, in orders that leave any of them
behind for as long as the barriers let it be.  Whatever the order, every role has to get through its share, and has to find in shared
memory what it expects there."""
import random

import pytest


class Barrier:
    """Completes a phase when `count` have arrived and no bytes are outstanding; a wait for a parity is answered by one bit."""

    def __init__(self, count):
        self.count, self.left, self.bytes, self.phase = count, count, 0, 0

    def arrive(self, expect=0):
        assert self.left > 0, "more arrivals than a phase has"
        self.left -= 1
        self.bytes += expect
        self.turn()

    def landed(self):
        self.bytes -= 1
        self.turn()

    def turn(self):
        if self.left == 0 and self.bytes == 0:
            self.phase, self.left = self.phase + 1, self.count

    def through(self, parity):
        return (self.phase & 1) != parity


N_BARS, SCALES = 8, 8
SOFTMAX, WIDENING = 2, 2          # warps of a row tile, and widening ones (what matters is that there are several)


class Cta:
    """One CTA's share: segments of (chunks, two tiles of different rows).  Of a tile's softmax warps the last has no rows."""

    def __init__(self, share, e4m3, one, head_128, softmax_counts, rng):
        self.e4m3, self.rng = e4m3, rng
        few = e4m3 and head_128 and not one
        self.nk = (3 if few else 4) if e4m3 else (3 if one else 2)
        self.nv = 2 if e4m3 else 3
        self.nr = 3 if few else 4
        self.softmax_counts = softmax_counts
        self.segments, n = [], 0
        for chunks, dual in share:
            self.segments.append((n, chunks, dual))
            n += chunks
        self.q_full, self.q_wide = Barrier(1), Barrier(WIDENING)
        self.q_empty = Barrier(2 + (2 * SOFTMAX if softmax_counts else 0))
        bars = lambda count, n=N_BARS: [Barrier(count) for _ in range(n)]  # noqa: E731
        self.k_full, self.k_empty, self.v_full, self.v_empty = bars(1), bars(2), bars(WIDENING if e4m3 else 1), bars(2)
        self.raw_full, self.raw_empty = bars(1, self.nr), bars(WIDENING, self.nr)
        pairs = lambda count: [[Barrier(count), Barrier(count)] for _ in range(2)]  # noqa: E731
        self.s_full, self.p_full = pairs(1), pairs(SOFTMAX)
        self.o_step, self.o_done, self.o_free = bars(1, 2), bars(1, 2), bars(SOFTMAX, 2)
        # what is in shared and tensor memory
        self.q = self.shift = None
        self.brief = [None, None]
        self.k, self.v, self.raw, self.scale = [None] * self.nk, [None] * self.nv, [None] * self.nr, [None] * SCALES
        self.o = [None, None]
        self.copies = []                                  # in flight, in any order
        self.queue = [[], []]                             # contractions and completions of each issuer, in order
        self.roles = [self.load_kv(), self.load_q(), self.issue(0), self.issue(1)]
        self.roles += [self.softmax(x, w) for x in range(2) for w in range(SOFTMAX)]
        if e4m3:
            self.roles += [self.widen(w) for w in range(WIDENING)]

    # chunks of a segment that tile x takes
    @staticmethod
    def chunks_of(segment, x):
        n0, chunks, dual = segment
        return [n for n in range(n0, n0 + chunks) if dual or (n & 1) == x]

    def copy(self, store, at, what, bar):
        def land():
            store[at] = what
            bar.landed()
        bar.arrive(expect=1)
        store[at] = None
        self.copies.append(land)

    def load_kv(self):
        for n0, chunks, _ in self.segments:
            for n in range(n0, n0 + chunks):
                if n >= self.nk:
                    yield self.k_empty[(n - self.nk) % N_BARS], (n - self.nk) // N_BARS & 1
                self.scale[n % SCALES] = n
                self.copy(self.k, n % self.nk, n, self.k_full[n % N_BARS])
                if self.e4m3:
                    if n >= self.nr:
                        yield self.raw_empty[n % self.nr], (n // self.nr - 1) & 1
                    self.copy(self.raw, n % self.nr, n, self.raw_full[n % self.nr])
                else:
                    if n >= self.nv:
                        yield self.v_empty[(n - self.nv) % N_BARS], (n - self.nv) // N_BARS & 1
                    self.copy(self.v, n % self.nv, n, self.v_full[n % N_BARS])

    def load_q(self):
        for s, _ in enumerate(self.segments):
            if s > 0:
                yield self.q_empty, (s - 1) & 1
            self.brief[s & 1] = s

            def land(s=s):
                self.q = s
                self.q_full.landed()
            self.q = None
            self.q_full.arrive(expect=1)
            self.copies.append(land)
        last = len(self.segments)
        yield self.q_empty, (last - 1) & 1
        self.brief[last & 1] = last
        self.q_full.arrive()

    def issue(self, x):
        q_phase = p_phase = o_phase = 0
        again, queue = False, self.queue[x]
        for s in range(len(self.segments) + 1):
            yield self.q_full, q_phase
            assert self.brief[q_phase] == s
            if s == len(self.segments):
                return
            if self.e4m3:
                yield self.q_wide, q_phase
            q_phase ^= 1
            dual, chunks = self.segments[s][2], self.chunks_of(self.segments[s], x)
            for j in range(len(chunks) + 1 if chunks else 0):
                for h in range(2):
                    if j > 0:
                        before = chunks[j - 1]
                        if h == 0:
                            yield self.v_full[before % N_BARS], before // N_BARS & 1
                            if j == 1 and again:
                                yield self.o_free[x], o_phase
                                o_phase ^= 1
                        yield self.p_full[x][h], p_phase
                        first, last = j == 1 and h == 0, j == len(chunks) and h == 1

                        def add(before=before, first=first, s=s):
                            assert self.v[before % self.nv] == before, "V is another chunk's"
                            assert first or self.o[x] == s
                            self.o[x] = s
                        queue.append(add)
                        queue.append(self.o_step[x].arrive)
                        if h == 1:
                            queue += [self.v_empty[before % N_BARS].arrive] * (1 if dual else 2)
                            if last:
                                queue.append(self.o_done[x].arrive)
                    if j < len(chunks):
                        n = chunks[j]
                        if h == 0:
                            yield self.k_full[n % N_BARS], n // N_BARS & 1

                        def multiply(n=n, s=s):
                            assert self.k[n % self.nk] == n and self.q == s, "K or Q is another's"
                            assert not self.e4m3 or self.shift == s
                        queue.append(multiply)
                        queue.append(self.s_full[x][h].arrive)
                        if h == 1:
                            queue += [self.k_empty[n % N_BARS].arrive] * (1 if dual else 2)
                if j > 0:
                    p_phase ^= 1
            if chunks:
                queue.append(self.q_empty.arrive)
            else:
                self.q_empty.arrive()
            again = again or bool(chunks)

    def softmax(self, x, w):
        sn = o_segs = 0
        rows = w + 1 < SOFTMAX
        for s in range(len(self.segments) + 1):
            yield self.q_full, s & 1
            assert self.brief[s & 1] == s, "another segment's description"
            if s == len(self.segments):
                return
            if rows and self.e4m3:
                yield self.q_wide, s & 1
                assert self.shift == s, "another segment's shift"
            if self.softmax_counts:
                self.q_empty.arrive()
            chunks = self.chunks_of(self.segments[s], x)
            for i in range(2 * len(chunks)):
                n, h = chunks[i >> 1], i & 1
                yield self.s_full[x][h], sn >> 1 & 1
                if rows:
                    if self.e4m3:
                        yield self.k_full[n % N_BARS], n // N_BARS & 1
                        assert self.scale[n % SCALES] == n, "another chunk's scales"
                    if i >= 1 and self.rng.random() < 0.5:
                        yield self.o_step[x], (sn - 1) & 1
                        assert self.o[x] == s
                self.p_full[x][h].arrive()
                sn += 1
            if chunks:
                yield self.o_done[x], o_segs & 1
                o_segs += 1
                if rows:
                    for _ in range(4):
                        yield None                        # the output's way out takes its time
                        assert self.o[x] == s, "O has been written over"
                self.o_free[x].arrive()

    def widen(self, w):
        for s, segment in enumerate(self.segments):
            yield self.q_full, s & 1
            assert self.brief[s & 1] == s
            self.shift = s
            self.q_wide.arrive()
            for n in range(segment[0], segment[0] + segment[1]):
                yield self.raw_full[n % self.nr], n // self.nr & 1
                gone = n - self.nv
                if gone >= 0:
                    yield self.v_empty[gone % N_BARS], gone // N_BARS & 1
                assert self.raw[n % self.nr] == n and self.scale[n % SCALES] == n
                self.v[n % self.nv] = n
                self.v_full[n % N_BARS].arrive()
                self.raw_empty[n % self.nr].arrive()
        yield self.q_full, len(self.segments) & 1

    def run(self):
        """Whether every role gets through: some of them, another choice now and then, only move when nothing else can."""
        rng, alive = self.rng, {i: r for i, r in enumerate(self.roles)}
        waits = {i: next(r, StopIteration) for i, r in alive.items()}
        slow = set()
        while True:
            for i in [i for i, w in waits.items() if w is StopIteration]:
                del waits[i], alive[i]
            if not alive:
                return True
            if rng.random() < 0.02:
                slow = set(rng.sample(range(len(self.roles) + 3), rng.randint(0, 4)))
            ready = [i for i, w in waits.items() if w is None or w[0].through(w[1])]
            queues = [i for i in range(2) if self.queue[i]]
            moves = [(i, "role") for i in ready] + [(len(self.roles) + i, "queue") for i in queues]
            moves += [(len(self.roles) + 2, "copy")] if self.copies else []
            if not moves:
                return False
            fast = [m for m in moves if m[0] not in slow]
            who, kind = rng.choice(fast or moves)
            if kind == "role":
                waits[who] = next(alive[who], StopIteration)
            elif kind == "queue":
                self.queue[who - len(self.roles)].pop(0)()
            else:
                self.copies.pop(rng.randrange(len(self.copies)))()


SHARES = [[(1, False)] * 9, [(3, False), (1, False)], [(2, False), (1, False), (1, False), (2, False)], [(1, True)] * 6, [(11, True), (1, False), (1, True)],
          [(14, True)], [(40, False)], [(23, True)], [(5, False), (1, False), (7, True), (1, False), (1, False), (30, False)]]


def shares(rng, one):
    for share in SHARES + [[(rng.choice([1, 1, 1, 2, 3, 5, 17]), rng.random() < 0.3) for _ in range(rng.randint(1, 12))] for _ in range(8)]:
        yield [(chunks, dual and not one) for chunks, dual in share]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("head_128", [False, True])
def test_every_role_gets_through(e4m3, one, head_128):
    rng = random.Random(int(e4m3) * 4 + int(one) * 2 + int(head_128))
    for share in shares(rng, one):
        for _ in range(5):
            assert Cta(share, e4m3, one, head_128, True, rng).run(), share


def runs(*args):
    try:
        return Cta(*args).run()
    except AssertionError:
        return False


@pytest.mark.parametrize("e4m3", [False, True])
def test_the_model_sees_a_barrier_that_is_passed_twice(e4m3):
    """With the softmax warps left out of what Q waits for, the model finds orders in which one of them waits for good, or reads another
    segment's shift; not where there is one segment."""
    rng = random.Random(1)
    fails = lambda share: not all(runs(share, e4m3, True, True, False, rng) for _ in range(100))  # noqa: E731
    assert fails([(3, False), (1, False)]) and fails([(1, False)] * 9) and fails(SHARES[2]) and not fails([(40, False)])
