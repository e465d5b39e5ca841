"""The waits of the chunk-attention kernel, as a discrete model of its roles: copies, conversion of 8-bit codes, matrix
products (one queue, in order), two softmax halves of four warps, queries.  A parity wait passes exactly when the barrier's
current phase has the other parity, so a barrier two phases from the expected one either lets the wait through too early
or holds it for ever; the model raises for the first and finds the second because nothing is left to happen.  Durations
are drawn at random over a wide range, since no order may depend on them.  A wait that runs out makes every role leave: each
notices that at its next wait that does not pass, after a while of its own.

The model's list of waits is compared with the kernel's source, so that neither is changed alone."""
import heapq
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_15763_b200", "csrc", "hos_attn_chunk.cu")


class Stuck(Exception):
    pass


class WrongPhase(Exception):
    pass


class Bar:
    def __init__(self, name, count):
        self.name, self.count, self.have, self.done = name, count, 0, 0

    def arrive(self):
        self.have += 1
        if self.have == self.count:
            self.have, self.done = 0, self.done + 1


class Model:
    """tiles: (steps, halves) of the tiles of one CTA's share."""

    def __init__(self, tiles, stages, q8, rng, slow=None, wait_for_k_stage=False, gives_up_at=None, vote=True):
        self.tiles, self.stages, self.q8, self.rng, self.slow = tiles, stages, q8, rng, slow or {}
        self.bufs, self.wait_for_k_stage = stages // 2 + 1, wait_for_k_stage
        n = 4 if q8 else 1
        self.kv_full = [Bar(f"kv_full{i}", n) for i in range(stages)]
        self.kv_free = [Bar(f"kv_free{i}", 1) for i in range(stages)]
        self.raw_full = [Bar(f"raw_full{i}", 1) for i in range(stages)] if q8 else self.kv_full
        self.scales_full = [Bar(f"scales_full{i}", 4) for i in range(self.bufs)]
        self.q_full, self.q_free, self.s_full, self.o_done = ([Bar(f"{k}{h}", 1) for h in (0, 1)] for k in ("q_full", "q_free", "s_full", "o_done"))
        self.p_half, self.p_ready = ([Bar(f"{k}{h}", 4) for h in (0, 1)] for k in ("p_half", "p_ready"))
        self.named, self.named_gen, self.votes, self.outcome = 0, 0, [], {}
        self.scale_of, self.stage_of = [None] * self.bufs, [None] * stages
        self.now, self.heap, self.n, self.waiting = 0.0, [], 0, []
        self.queue_free = 0.0
        self.gave_up, self.gives_up_at, self.vote = False, gives_up_at, vote

    # --- clockwork ---
    def later(self, t, what):
        self.n += 1
        heapq.heappush(self.heap, (t, self.n, what))

    def time(self, kind):
        return self.slow.get(kind, 1.0) * self.rng.choice((0.1, 1.0, 10.0)) * self.rng.random()

    def resume(self, co, value=None):
        try:
            while True:
                step = co.send(value)
                if step[0] == "sleep":
                    self.later(self.now + step[1], lambda: self.resume(co))
                    return
                if not self.passes(step):
                    self.waiting.append((step, co))
                    if self.gave_up:
                        self.notice(step, co)
                    return
                value = True
        except StopIteration:
            pass

    def notice(self, step, co):
        """The waiting role sees some time later that another has given up, unless its wait has passed by then."""
        def look():
            for i, (s, c) in enumerate(self.waiting):
                if s is step and c is co and s[0] == "wait":
                    del self.waiting[i]
                    self.resume(co, False)
                    return
        self.later(self.now + 20.0 * self.rng.random(), look)

    def give_up(self):
        self.gave_up = True
        for step, co in list(self.waiting):
            self.notice(step, co)

    def passes(self, step):
        if step[0] == "named":
            return self.named_gen > step[1]
        _, bar, parity, want = step
        if (bar.done & 1) == parity:
            return False
        if bar.done != want:
            raise WrongPhase(f"{bar.name}: {bar.done} phases done where {want} were meant")
        return True

    def run(self):
        roles = [self.copies(), self.products(), self.queries(0), self.queries(1)]
        roles += [self.softmax(h) for h in (0, 1) for _ in range(4)] + ([self.convert() for _ in range(4)] if self.q8 else [])
        left = [len(roles)]

        def counted(role):
            yield from role
            left[0] -= 1
        for r in roles:
            self.later(0.0, lambda co=counted(r): self.resume(co))
        if self.gives_up_at is not None:
            self.later(self.gives_up_at, self.give_up)
        while self.heap:
            self.now, _, what = heapq.heappop(self.heap)
            what()
            again = True
            while again:
                again = False
                for i, (step, co) in enumerate(self.waiting):
                    if self.passes(step):
                        del self.waiting[i]
                        self.resume(co, True)
                        again = True
                        break
        if left[0]:
            raise Stuck(", ".join(sorted({s[1].name for s, _ in self.waiting if s[0] == "wait"})))

    def issue(self, kind, then):
        """A matrix product or commit: runs after everything issued before it."""
        self.queue_free = max(self.queue_free, self.now) + (self.time(kind) if kind else 0.0)
        self.later(self.queue_free, then)

    @staticmethod
    def wait(bar, index, flipped=False):
        """Waits for phase number `index`; flipped: for the one before (a stage that starts out free)."""
        return ("wait", bar, (index & 1) ^ (1 if flipped else 0), index + (0 if flipped else 1))

    # --- roles, in the kernel's order ---
    def copies(self):
        item = 0
        for blocks, _ in self.tiles:
            for _ in range(2 * blocks):
                stage, rnd = item % self.stages, item // self.stages
                if not (yield self.wait(self.kv_free[stage], rnd, flipped=True)):
                    return

                def landed(stage=stage, item=item):
                    self.stage_of[stage] = item
                    self.raw_full[stage].arrive()
                self.later(self.now + self.time("copy"), landed)
                item += 1
                yield ("sleep", self.time("issue"))

    def convert(self):
        for block in range(sum(b for b, _ in self.tiles)):
            item = 2 * block
            ok = yield self.wait(self.raw_full[item % self.stages], item // self.stages)
            if not self.vote and not ok:
                return
            yield ("sleep", self.time("scales"))
            if ok:
                self.scale_of[block % self.bufs] = block
            self.scales_full[block % self.bufs].arrive()
            for i in (item, item + 1):
                if i > item:
                    ok = True
                if ok:
                    ok = yield self.wait(self.raw_full[i % self.stages], i // self.stages)
                if not self.vote and not ok:
                    return
                yield ("sleep", self.time("codes"))
                gen = self.named_gen
                self.named += 1
                self.votes.append(ok)
                if self.named == 4:
                    self.outcome[gen], self.votes = all(self.votes), []
                    self.named, self.named_gen = 0, gen + 1
                yield ("named", gen)
                if not self.outcome[gen]:
                    return
                yield ("sleep", self.time("codes"))
                self.kv_full[i % self.stages].arrive()

    def products(self):
        item = tile = 0
        block = [0, 0]

        def meant(i):
            if self.stage_of[i % self.stages] != i:
                raise WrongPhase(f"a product of item {i} reads item {self.stage_of[i % self.stages]}")
        for blocks, halves in self.tiles:
            for h in (0, 1):
                if not (yield self.wait(self.q_full[h], tile)):
                    return
            if not (yield self.wait(self.kv_full[item % self.stages], item // self.stages)):
                return
            for h in range(halves):
                self.issue("qk", lambda i=item: meant(i))
                self.issue(None, self.s_full[h].arrive)
            self.issue(None, self.kv_free[item % self.stages].arrive)
            if blocks == 1:
                for h in (0, 1):
                    self.issue(None, self.q_free[h].arrive)
            for b in range(blocks):
                vi, ki, more = item + 1, item + 2, b + 1 < blocks
                if not (yield self.wait(self.kv_full[vi % self.stages], vi // self.stages)):
                    return
                if more:
                    if not (yield self.wait(self.kv_full[ki % self.stages], ki // self.stages)):
                        return
                for h in range(halves):
                    if not (yield self.wait(self.p_half[h], block[h])):
                        return
                    self.issue("pv", lambda i=vi: meant(i))
                    if not (yield self.wait(self.p_ready[h], block[h])):
                        return
                    block[h] += 1
                    self.issue("pv", lambda i=vi: meant(i))
                    if more:
                        self.issue("qk", lambda i=ki: meant(i))
                        self.issue(None, self.s_full[h].arrive)
                    else:
                        self.issue(None, self.o_done[h].arrive)
                self.issue(None, self.kv_free[vi % self.stages].arrive)
                if more:
                    self.issue(None, self.kv_free[ki % self.stages].arrive)
                if b + 2 == blocks:
                    for h in (0, 1):
                        self.issue(None, self.q_free[h].arrive)
                item += 2
                yield ("sleep", self.time("issue"))
            tile += 1

    def queries(self, h):
        for tile in range(len(self.tiles)):
            if not (yield self.wait(self.q_free[h], tile, flipped=True)):
                return
            yield ("sleep", self.time("queries"))
            self.q_full[h].arrive()

    def softmax(self, h):
        block = mine = tiles = 0
        for blocks, halves in self.tiles:
            if h >= halves:
                block += blocks
                continue
            for _ in range(blocks):
                if self.wait_for_k_stage:
                    if not (yield self.wait(self.kv_full[2 * block % self.stages], 2 * block // self.stages)):
                        return
                if not (yield self.wait(self.s_full[h], mine)):
                    return
                mine += 1
                if self.q8 and not self.wait_for_k_stage:
                    if not (yield self.wait(self.scales_full[block % self.bufs], block // self.bufs)):
                        return
                if self.q8 and self.scale_of[block % self.bufs] != block:
                    raise WrongPhase("scales of another step")
                yield ("sleep", self.time("weights"))
                if not self.q8 and h == 0:
                    if not (yield self.wait(self.kv_full[(2 * block + 1) % self.stages], (2 * block + 1) // self.stages)):
                        return
                self.p_half[h].arrive()
                yield ("sleep", self.time("weights"))
                if self.q8 and self.scale_of[block % self.bufs] != block:
                    raise WrongPhase("scales of another step")
                self.p_ready[h].arrive()
                block += 1
            if not (yield self.wait(self.o_done[h], tiles)):
                return
            tiles += 1
            yield ("sleep", self.time("output"))


def test_waits_of_the_source():
    text = open(SOURCE).read()
    marks = ["softmax and output =", "K and V by TMA =", "the products =", "queries =", "K and V of an 8-bit cache =", "tcgen05.dealloc"]
    at = [text.index(m) for m in marks]
    assert at == sorted(at)
    waits = [re.findall(r"bar_wait\((\w+)\(", text[a:b]) for a, b in zip(at, at[1:])]
    assert waits == [
        ["kv_full", "s_full", "scales_full", "o_done"],           # kv_full: in clear_v, V of a step with hidden tokens, half 0, 16-bit
        ["kv_free"],
        ["q_full", "kv_full", "kv_full", "kv_full", "p_half", "p_ready"],
        ["q_free"],
        ["raw_full", "raw_full"],                                 # in convert; of the step's K before its scales are written
    ]
    convert = text[at[4]:at[5]]
    # the named barrier has no limit: all four warps come to it, whatever became of their waits, and leave on the common vote only
    assert "bar.sync" not in convert and convert.count("all_of_four_warps(") == 1
    loop = convert[convert.index("for (int block"):]
    assert "break" not in loop[:loop.index("!convert(item")] and "return" not in convert[convert.index("auto convert"):convert.index("if (!all_of_four_warps")]
    assert convert.index("bar_arrive(scales_full(") < convert.index("!convert(item")
    assert convert.index("fence_async_smem") < convert.index("bar_arrive(kv_full(")


SHAPES = [[(b, 2) for b in (1, 2, 3, 4, 7, 1, 1, 5, 3)], [(3, 2)] * 12, [(1, 1)] * 9 + [(2, 2)] * 4, [(b, 1 + b % 2) for b in range(1, 12)],
          [(20, 1), (1, 2), (9, 1), (9, 1), (1, 2), (30, 2)]]


@pytest.mark.parametrize("stages", [4, 8])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("slow", [{}, {"output": 100.0}, {"weights": 50.0}, {"copy": 50.0}, {"qk": 30.0, "pv": 30.0}, {"codes": 30.0},
                                  {"queries": 60.0}, {"scales": 40.0}], ids=lambda s: "+".join(s) or "even")
def test_no_order_depends_on_time(stages, q8, slow):
    for seed in range(12):
        for tiles in SHAPES:
            Model(tiles, stages, q8, random.Random(seed), slow).run()


def test_the_model_finds_a_wait_on_a_reused_stage():
    """Waiting for K's stage in the softmax warps stops everything once a tile's output takes long."""
    with pytest.raises((Stuck, WrongPhase)):
        for seed in range(20):
            Model([(3, 2)] * 6, 4, True, random.Random(seed), {"output": 100.0}, wait_for_k_stage=True).run()
    with pytest.raises(Stuck):
        Model([(3, 2)] * 6, 4, True, random.Random(0), {"output": 1e4}, wait_for_k_stage=True).run()


@pytest.mark.parametrize("q8", [False, True])
def test_every_role_leaves_once_a_wait_has_run_out(q8):
    for seed in range(150):
        rng = random.Random(seed)
        Model(SHAPES[seed % len(SHAPES)], rng.choice((4, 8)), q8, rng, {rng.choice(("copy", "output", "codes", "qk")): 30.0},
              gives_up_at=rng.random() * 600.0).run()


def test_the_model_finds_warps_that_leave_before_the_named_barrier():
    with pytest.raises(Stuck):
        for seed in range(300):
            rng = random.Random(seed)
            Model(SHAPES[seed % len(SHAPES)], 4, True, rng, {"copy": 30.0}, gives_up_at=rng.random() * 600.0, vote=False).run()


def test_a_wait_that_ran_out_is_reported_whoever_waited():
    """After all roles have met again, from the flag they share, for every sequence of the share."""
    text = open(SOURCE).read()
    body = text[text.index("__global__"):text.index("// Tensor map of k or v")]
    assert len(re.findall(r"a\.kv\.status \+ \S+, HOS_ST_LIMIT", body)) == 1
    last = body.rindex("__syncthreads();")
    report = body.index("HOS_ST_LIMIT")
    assert last < body.index("if (*gave_up && threadIdx.x == 0 && a.kv.status)") < report < body.index("tcgen05.dealloc")
    assert "while (list.next(c, share));" in body[report:]
