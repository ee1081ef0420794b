"""The order of barriers in the bf16 attention to an encoder's states (csrc/attn_cross.cu, attn_cross_tc), as a model on the CPU.

One warp brings tiles of K and V through a ring of stages, one warp per tile of rows issues its products, and four warps per tile of rows take its
weights.  A wait names the parity of a phase, so a barrier that runs two phases ahead of a waiter stops everything for good: the model runs all parts
in random order, copies and products that land late and in any order they can, over random lists of items, and looks for that, and for a stage that does
not hold what a product reads.  It restates the kernel's loops and has to be changed along with them."""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count = self.pending = count
        self.phase = 0

    def arrive(self):
        self.pending -= 1
        assert self.pending >= 0
        if self.pending == 0:
            self.pending, self.phase = self.count, self.phase + 1

    def passed(self, parity):
        return (self.phase & 1) != parity


class Cursor:
    """The stages that hold K (from 0 on), or V (from 1 on): every other one."""

    def __init__(self, stage, stages):
        self.stage, self.phase, self.stages = stage, 0, stages

    def advance(self):
        self.stage += 2
        if self.stage >= self.stages:
            self.stage -= self.stages
            self.phase ^= 1


def run(items, tiles, stages, seed, forget=None):
    """items: (tiles of states, more than 128 rows, a part of a block only).  forget: a step of the kernel's that is left out.  True: all ended."""
    rng = random.Random(seed)
    q_full, s_full, p_ready, o_full, turn = ([Barrier(1) for _ in range(2)] for _ in range(5))
    kv_full, kv_free = [Barrier(1) for _ in range(stages)], [Barrier(2) for _ in range(stages)]
    in_stage, in_flight, products = {}, [], ([], [])                # products of a warp end in the order of their issue
    met = {"count": 0, "generation": 0}                             # the barrier of both tiles' threads

    def loader():
        pos = 0
        for count, _, _ in items:
            for _ in range(2 * count):
                stage, use = pos % stages, pos // stages
                if use > 0:
                    yield kv_free[stage], (use - 1) & 1
                in_stage[stage] = pos
                in_flight.append(kv_full[stage])
                pos += 1
                yield None

    def issuer(t):
        kc, vc = Cursor(0, stages), Cursor(1, stages)

        def landed(c):
            return kv_full[c.stage], c.phase

        def let_pass(c):
            yield landed(c)
            kv_free[c.stage].arrive()
            c.advance()

        q_phase = q1_phase = p_phase = turn_phase = before = 0
        first_turn = t == 0
        for count, rows, _ in items:
            two = tiles == 2 and rows
            both = tiles == 2 and not two
            yield q_full[0], q_phase
            q_phase ^= 1
            if two:
                if t == 1:
                    yield q_full[1], q1_phase
                q1_phase ^= 1
            step, mine = (2, (count - t + 1) // 2) if both else (1, count)
            turns = ((count + 1) // 2 if both else count) + 1
            if both and t == 1:
                yield from let_pass(kc)
                yield from let_pass(vc)
            for j in range(-1, turns - 1):
                value, score = 0 <= j < mine, j < mine - 1
                if score:
                    if step == 2 and j >= 0:
                        yield from let_pass(kc)
                    if j < 0:
                        yield landed(kc)
                if value:
                    yield landed(vc)
                    yield p_ready[t], p_phase
                    p_phase ^= 1
                if tiles == 2 and not first_turn:
                    yield turn[t], turn_phase
                    turn_phase ^= 1
                first_turn = False
                if value:
                    assert in_stage[vc.stage] == 2 * (before + (t + 2 * j if both else j)) + 1
                    products[t].append(kv_free[vc.stage])
                    if tiles == 1:
                        kv_free[vc.stage].arrive()
                    if j == mine - 1:
                        products[t].append(o_full[t])
                    vc.advance()
                    if step == 2 and j < mine - 1:
                        yield from let_pass(vc)
                if score:
                    if j >= 0:
                        yield landed(kc)
                    assert in_stage[kc.stage] == 2 * (before + (t + 2 * (j + 1) if both else j + 1))
                    products[t].append(s_full[t])
                    kc.advance()
                if tiles == 2:
                    turn[1 - t].arrive()
                yield None
            if both and (count - t) % 2 == 0 and count > t and forget != "the other tile's last stages":
                yield from let_pass(kc)
                yield from let_pass(vc)
            before += count

    def meet():
        generation = met["generation"]
        met["count"] += 1
        if met["count"] == 2:
            met["count"], met["generation"] = 0, generation + 1
        while met["generation"] == generation:
            yield "others"

    def weights(t):
        s_used = o_used = before = 0
        for count, rows, part in items:
            two = tiles == 2 and rows
            both = tiles == 2 and not two
            if t == 0 or two:
                q_full[t].arrive()
            blocks = 0
            for j in range(t if both else 0, count if t == 0 or tiles == 2 else 0, 2 if both else 1):
                yield s_full[t], s_used & 1
                s_used += 1
                stage = 2 * (before + j) % stages
                kv_free[stage].arrive()                             # K has been used
                if tiles == 1:
                    kv_free[stage].arrive()
                if rng.random() < 0.3:                              # masked states: their values are set to zero in the stage
                    pos = 2 * (before + j) + 1
                    yield kv_full[pos % stages], pos // stages & 1
                    assert in_stage[pos % stages] == pos
                p_ready[t].arrive()
                blocks += 1
                yield None
            before += count
            if blocks:
                yield o_full[t], o_used & 1
                o_used += 1
            if both and count > 1:                                  # two results of the same rows are added
                for _ in range(3):
                    yield from meet()
            if part:
                for _ in range(2):
                    yield from meet()

    parts = {"loader": loader(), "weights 0": weights(0), "weights 1": weights(1)}
    for t in range(tiles):
        parts["issuer %d" % t] = issuer(t)
    waits = dict.fromkeys(parts)
    idle = 0
    while parts:
        moved = False
        for name in rng.sample(list(parts), len(parts)):
            at = waits[name]
            if isinstance(at, tuple) and not at[0].passed(at[1]):
                continue
            for _ in range(rng.choice((1, 1, 3))):
                try:
                    at = waits[name] = next(parts[name])
                except StopIteration:
                    del parts[name], waits[name]
                    moved = True
                    break
                moved = moved or at != "others"
                if at == "others" or isinstance(at, tuple) and not at[0].passed(at[1]):
                    break
        if in_flight and rng.random() < 0.7:
            in_flight.pop(rng.randrange(len(in_flight))).arrive()
            moved = True
        for queue in products:
            if queue and rng.random() < 0.7:
                queue.pop(0).arrive()
                moved = True
        idle = 0 if moved or in_flight or any(products) else idle + 1
        if idle > 20:
            return False
    return True


def lists(seed):
    rng = random.Random(seed)
    return [(rng.choice((1, 1, 2, 3, 4, 5, 8)), rng.random() < 0.5, rng.random() < 0.3) for _ in range(rng.randint(1, 6))]


@pytest.mark.parametrize("tiles,stages", [(2, 5), (2, 8), (1, 5)])
def test_every_list_ends(tiles, stages):
    for seed in range(1000):
        assert run(lists(seed), tiles, stages, seed), (seed, lists(seed))


def test_the_model_sees_a_missed_phase():
    def ends(seed):
        try:
            return run(lists(seed), 2, 5, seed, forget="the other tile's last stages")
        except AssertionError:                                      # a stage that holds something else
            return False

    assert not all(ends(seed) for seed in range(40))
