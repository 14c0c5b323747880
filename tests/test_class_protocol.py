"""The hand-over of rows inside ``k_class_ring`` (csrc/lrgd_class.cuh), replayed on the CPU under random schedules: the copying warps, the
teams, and the warps that work out a row's numbers, in clusters of CTAs.  An mbarrier's wait knows a phase only by its parity, so every
wait that returns has to return for the phase that is meant, no place may be overwritten while somebody still reads it, and all have to
come to their end."""
import random

import pytest

TEAM_WARPS, NUMBERS, ROWS = 3, 4, 4                 # (three warps a team instead of up to nine: fewer steps, the same protocol)


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.phase, self.tx = count, count, 0, 0

    def settle(self):
        if self.left == 0 and self.tx == 0:
            self.phase, self.left = self.phase + 1, self.count

    def arrive(self, tx=0):
        assert self.left > 0, "more arrivals than the phase has"
        self.left, self.tx = self.left - 1, self.tx + tx
        self.settle()

    def complete(self, tx):
        self.tx -= tx
        self.settle()


def wait(bar, parity, phase):
    """Waits as the hardware does (the phase with this parity is complete); `phase` is the one that is meant."""
    while bar.phase & 1 == parity & 1:
        yield "waits"
    assert bar.phase == phase + 1, f"returned for phase {bar.phase - 1}, meant {phase}"


class Cta:
    def __init__(self, teams, depth):
        self.full = [[Barrier(1) for _ in range(depth)] for _ in range(teams)]
        self.free = [[Barrier(TEAM_WARPS) for _ in range(depth)] for _ in range(teams)]
        self.ring = [[None] * depth for _ in range(teams)]
        self.summed, self.ready, self.written = ([Barrier(n) for _ in range(ROWS)] for n in (TEAM_WARPS, 1, TEAM_WARPS))
        self.joined = [Barrier(1) for _ in range(2 * ROWS)]
        self.sums, self.row, self.cta_sum = [{} for _ in range(ROWS)], [None] * ROWS, [{} for _ in range(2 * ROWS)]
        self.inflight, self.done = [], {}


def copier(c, teams, team, mine, stages, depth, grad):
    copies = 0
    for k in range(team, mine, teams):
        n = stages(k)
        for i in [*range(n), *range(max(0, n - depth) if grad else 0)]:
            slot, lap = copies % depth, copies // depth
            if lap:
                yield from wait(c.free[team][slot], lap - 1, lap - 1)
            c.full[team][slot].arrive(tx=1)
            c.inflight.append((team, slot, (k, i)))
            copies += 1
            yield


def passes(c, teams, team, warp, mine, stages, depth, grad):
    used = 0
    for k in range(team, mine, teams):
        n, at, lap = stages(k), k % ROWS, k // ROWS
        dropped = max(0, n - depth) if grad else n
        for i in range(n):
            slot = used % depth
            yield from wait(c.full[team][slot], used // depth, used // depth)
            assert c.ring[team][slot] == (k, i)
            yield
            assert c.ring[team][slot] == (k, i), "overwritten while it was read"
            if i < dropped:
                c.free[team][slot].arrive()
            used += 1
        if not grad and k >= ROWS:
            yield from wait(c.ready[at], lap - 1, lap - 1)
        c.sums[at][warp] = k
        c.summed[at].arrive()
        yield
        if not grad:
            continue
        yield from wait(c.ready[at], lap, lap)
        assert c.row[at] == k
        for i in range(dropped, n):
            slot = (used - n + i) % depth
            assert c.ring[team][slot] == (k, i), "a stage was not kept between the passes"
            yield
            c.free[team][slot].arrive()
        for i in range(dropped):
            slot = used % depth
            yield from wait(c.full[team][slot], used // depth, used // depth)
            assert c.ring[team][slot] == (k, i)
            yield
            c.free[team][slot].arrive()
            used += 1
        c.written[at].arrive()
        yield


def numbers(ctas, rank, h, mine, grad):
    c, C = ctas[rank], len(ctas)
    for k in range(h, mine, NUMBERS):
        at, lap = k % ROWS, k // ROWS
        yield from wait(c.summed[at], lap, lap)
        assert all(v == k for v in c.sums[at].values()) and len(c.sums[at]) == TEAM_WARPS
        yield
        if C > 1:
            at2, lap2 = k % (2 * ROWS), k // (2 * ROWS)
            c.joined[at2].arrive(tx=C)
            for peer in ctas:                       # a message: the data, then the count on the peer's barrier
                yield
                peer.cta_sum[at2][rank] = k
                peer.joined[at2].complete(1)
            yield from wait(c.joined[at2], lap2, lap2)
            yield
            assert all(v == k for v in c.cta_sum[at2].values()) and len(c.cta_sum[at2]) == C, "a message was overwritten before it was read"
        c.row[at] = k
        c.ready[at].arrive()
        yield
        if grad:
            yield from wait(c.written[at], lap, lap)
        c.done[k] = c.done.get(k, 0) + 1


@pytest.mark.parametrize("teams", [2, 4])
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("C,depth,stages", [(1, 3, 1), (1, 3, 3), (1, 4, 2), (1, 3, 5), (1, 2, 7), (2, 3, 2), (4, 3, 1), (2, 3, 4), (4, 5, 3), (1, 3, 0),
                                            (2, 3, "ragged"), (1, 4, "ragged")])
def test_rows_are_handed_over(teams, grad, C, depth, stages):
    for seed in range(6):
        rng = random.Random(seed)
        mine = rng.choice([1, 2, 3, 9, 26])
        ctas = [Cta(teams, depth) for _ in range(C)]
        agents = []
        for r, c in enumerate(ctas):
            count = (lambda k, r=r: (k * 7 + r) % 6) if stages == "ragged" else (lambda k: stages)
            agents += [copier(c, teams, t, mine, count, depth, grad) for t in range(teams)]
            agents += [passes(c, teams, t, w, mine, count, depth, grad) for t in range(teams) for w in range(TEAM_WARPS)]
            agents += [numbers(ctas, r, h, mine, grad) for h in range(NUMBERS)]
        weight = [rng.choice([1, 1, 1, 10, 50]) for _ in agents]      # some are much faster than others
        alive, waiting = list(range(len(agents))), set()
        while alive:
            i = rng.choices(alive, [weight[j] for j in alive])[0]
            try:
                if next(agents[i]) == "waits":
                    waiting.add(i)
                else:
                    waiting.clear()
            except StopIteration:
                alive.remove(i)
                waiting.clear()
            for c in ctas:                          # copies land some time later, in any order
                if c.inflight and rng.random() < 0.5:
                    team, slot, what = c.inflight.pop(rng.randrange(len(c.inflight)))
                    c.ring[team][slot] = what
                    c.full[team][slot].complete(1)
                    waiting.clear()
            assert not alive or len(waiting) < len(alive) or any(c.inflight for c in ctas), "they wait for one another"
        assert all(c.done == {k: 1 for k in range(mine)} for c in ctas)
