"""The waits of the question kernel's byte rings, as a model on the CPU.

A barrier is waited for by the parity of a phase, and says yes if an odd number of phases lies between that one and the one under way.
That is right only for a waiter that knows the phase before to be complete.  The model runs the warp that asks for the bytes of half
steps and the pairs of warps that widen them in every order that their waits allow, bytes arriving in any order, and fails where a
pair goes on although its bytes are not there, or where nobody can go on."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2607_21599_b200", "csrc", "daf_page_attn.cu")


def _constants():
    text = open(SOURCE).read()
    stages = int(re.search(r"constexpr int kQStages = (\d+);", text).group(1))
    full = re.search(r"constexpr int kQFull = (\d+) \* kQStages;", text)
    assert re.search(r"const int turn = \(warp >> 1\) & 1", text) and re.search(r"for \(int t = turn; t < 2 \* n_t; t \+= 2\)", text), "two pairs in turn"
    return stages, stages * int(full.group(1)) if full else stages


def _run(stages, full, turns, steps, before):
    """Every reachable state of one piece of `steps` half steps behind one of `before`; the first fault, or None.

    A state: half steps asked for, which of them have arrived, where each pair is.  What is waited for are `full` barriers in turn for
    the bytes (`before` and what has arrived say how many phases each has completed) and one of `stages` slots to be free."""
    def phases(barrier, arrived):
        return sum(1 for t in range(before) if t % full == barrier) + sum(1 for t in arrived if t % full == barrier)

    def says_yes(barrier, use, arrived):
        start = sum(1 for t in range(before) if t % full == barrier)
        return (phases(barrier, arrived) & 1) != ((start + use) & 1)

    start = (0, frozenset(), tuple(range(turns)))
    seen, todo = {start}, [start]
    while todo:
        asked, arrived, at = state = todo.pop()
        nexts = []
        consumed = {t for k, pos in enumerate(at) for t in range(k, pos, turns)}
        if asked < steps and (asked < stages or asked - stages in consumed):
            nexts.append((asked + 1, arrived, at))
        nexts += [(asked, arrived | {t}, at) for t in range(asked) if t not in arrived]
        for k, t in enumerate(at):
            if t < steps and says_yes(t % full, t // full, arrived):
                if t not in arrived:
                    return f"half step {t} is taken before its bytes are there (asked for: {asked}, there: {sorted(arrived)}, pairs at {at})"
                nexts.append((asked, arrived, at[:k] + (t + turns,) + at[k + 1:]))
        if not nexts and any(t < steps for t in at):
            return f"nobody can go on: {state}"
        for s in nexts:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


def test_the_model_tells_right_from_wrong():
    assert _run(2, 2, 2, 8, 0) is None and _run(4, 4, 2, 10, 3) is None and _run(3, 3, 1, 9, 1) is None
    assert "is taken before its bytes are there" in _run(3, 3, 2, 10, 0)


@pytest.mark.parametrize("before", range(0, 13, 2))
@pytest.mark.parametrize("steps", [2, 4, 8, 14])
def test_bytes_are_there_when_they_are_widened(steps, before):
    stages, full = _constants()
    assert _run(stages, full, 2, steps, before) is None


# ---------------------------------------------------------------------------------------------------------- the whole kernel
class _Wrong(AssertionError):
    pass


class _Model:
    """The roles of the kernel as generators that yield what they wait for; buffers hold the name of what was put there last.

    Copies and products end some time after they are asked for, products of one warp in order.  A wait passes by parity, as on the
    device, with each barrier's parity at the begin of a piece from bar_uses' formula; passing ahead of its phase, a buffer that holds
    something else when it is read or while a product runs, and a standstill are faults."""
    CONSTS = 16

    def __init__(self, rng, stages, full):
        self.rng, self.stages, self.full = rng, stages, full
        self.count, self.here, self.done, self.base, self.odd = {}, {}, {}, {}, {}
        self.mem = {}
        for kv in range(2):
            self._bars(("st_full", kv), full, 1)
            self._bars(("st_empty", kv), stages, 2)
        for name, n, count in (("k_full", 2, 4), ("k_empty", 2, 2), ("v_full", 4, 2), ("v_empty", 4, 2), ("q_full", 2, 4), ("s_full", 2, 1),
                               ("o_full", 2, 1), ("c_full", self.CONSTS, 4)):
            self._bars((name,), n, count)
        for g in range(2):
            self._bars(("p_full", g), 2, 4)
            self._bars(("turn", g), 4, 1)

    def _bars(self, name, n, count):
        for i in range(n):
            b = name + (i,)
            self.count[b], self.here[b], self.done[b], self.odd[b] = count, 0, 0, 0

    def arrive(self, bar, n=1):
        for _ in range(n):
            self.here[bar] += 1
            if self.here[bar] == self.count[bar]:
                self.here[bar] = 0
                self.done[bar] += 1

    def passes(self, bar, phase):
        if (self.done[bar] & 1) == ((self.odd[bar] + phase) & 1):
            return False
        if self.done[bar] - self.base[bar] != phase + 1:
            raise _Wrong(f"{bar}: phase {phase} taken with {self.done[bar] - self.base[bar]} complete")
        return True

    def holds(self, where, what):
        if self.mem.get(where) != what:
            raise _Wrong(f"{where} holds {self.mem.get(where)}, not {what}")

    @staticmethod
    def uses(bar, n_t, pair, stages, full):
        """bar_uses of the kernel."""
        name, i = bar[0], bar[-1]
        if name == "st_full":
            return (2 * n_t - i + full - 1) // full
        if name == "st_empty":
            return (2 * n_t - i + stages - 1) // stages
        if name in ("k_full", "k_empty"):
            return (n_t - i + 1) >> 1
        if name in ("v_full", "v_empty"):
            return (n_t if i < 2 else 0) if pair else (n_t - (i >> 1) + 1) >> 1
        if name == "q_full":
            return 1
        if name == "turn":
            return n_t if pair else 0
        if name == "c_full":
            return (2 * n_t - i + 15) // 16
        g = bar[1]
        steps = n_t if pair else (n_t - g + 1) >> 1
        return min(steps, 1) if name == "o_full" else steps

    # ---- roles.  Yields a (barrier, phase), a function to become true, or None (anything may happen in between)
    def loader(self, kv, n_t):
        for t in range(2 * n_t):
            if t >= self.stages:
                yield ("st_empty", kv, t % self.stages), t // self.stages - 1
            self.copies.append((("stage", kv, t % self.stages), t, ("st_full", kv, t % self.full), self.rng.random() ** 4 + 0.003))
            yield None
            if kv == 0:
                self.mem["chunk", t % self.CONSTS] = t
                self.arrive(("c_full", t % self.CONSTS), 4)
                yield None

    def widener(self, kv, turn, which, n_t, pair):
        go = ("go", kv, turn)
        for t in range(turn, 2 * n_t, 2):
            step = t >> 1
            slot, use = (step & 1, step >> 1) if kv == 0 else (t & 1, step) if pair else (t & 3, step >> 1)
            if which == 0:
                yield ("st_full", kv, t % self.full), t // self.full
                if kv == 1:
                    yield ("c_full", t % self.CONSTS), t // self.CONSTS
                if step == 0 and (kv == 0 or not pair):
                    yield ("q_full", 0), 0
                    yield ("q_full", 1), 0
                if use > 0:
                    yield ("k_empty" if kv == 0 else "v_empty", slot), use - 1
            self.mem[go, which] = t
            yield lambda t=t: self.mem.get((go, 1 - which), -1) >= t
            self.holds(("stage", kv, t % self.stages), t)
            if kv == 1:
                self.holds(("chunk", t % self.CONSTS), t)
            yield None
            self.holds(("stage", kv, t % self.stages), t)
            for what, where in self.running:
                if where == (("k", slot) if kv == 0 else ("v", slot)):
                    raise _Wrong(f"{where} is written while {what} reads it")
            if kv == 0:
                self.mem["k", slot, t & 1, which] = step
                self.arrive(("k_full", slot))
            else:
                self.mem["v", slot, which] = t
                self.arrive(("v_full", slot))
            yield None
            self.arrive(("st_empty", kv, t % self.stages))
            yield None

    def products(self, g, n_t, pair):
        n_u = n_t if pair else (n_t - g + 1) >> 1
        if n_u == 0:
            return
        release = 1 if pair else 2

        def qk(step):
            buf = step & 1
            reads = [(("k", buf, half, w), step) for half in range(2) for w in range(2)]
            self.queue[g].append(("qk", ("k", buf), reads, [(("s", g), step)], [(("s_full", g), 1), (("k_empty", buf), release)]))

        yield ("q_full", g if pair else 0), 0
        yield ("k_full", 0 if pair else g), 0
        qk(0 if pair else g)
        for u in range(n_u):
            t = u if pair else 2 * u + g
            for half in range(2):
                slot = half if pair else 2 * g + half
                yield ("v_full", slot), u
                yield ("p_full", g, half), u
                reads = [(("v", slot, w), 2 * t + half) for w in range(2)] + [(("p", g, half, w), t) for w in range(4)]
                last = [(("o_full", g), 1)] if u + 1 == n_u and half == 1 else []
                self.queue[g].append(("pv", ("v", slot), reads, [(("o", g), t)], [(("v_empty", slot), release)] + last))
                yield None
            if u + 1 < n_u:
                step = t + (1 if pair else 2)
                yield ("k_full", step & 1), step >> 1
                qk(step)
                yield None

    def softmax(self, g, w, n_t, pair, valid):
        n_u = n_t if pair else (n_t - g + 1) >> 1
        self.arrive(("q_full", g))
        yield None
        for u in range(n_u):
            t = u if pair else 2 * u + g
            c0 = 2 * t % self.CONSTS
            if valid:
                yield ("c_full", c0), 2 * t // self.CONSTS
                yield ("c_full", c0 + 1), 2 * t // self.CONSTS
            yield ("s_full", g), u
            for half in range(2):
                if half == 0 and pair and (g == 1 or u > 0):
                    yield ("turn", g, w), u if g == 1 else u - 1
                if valid:
                    self.holds(("s", g), t)
                    self.holds(("chunk", c0), 2 * t)
                    self.holds(("chunk", c0 + 1), 2 * t + 1)
                    if half == 0 and u > 0:
                        self.holds(("o", g), t - (1 if pair else 2))      # the product before is complete: O may be scaled
                self.mem["p", g, half, w] = t
                self.arrive(("p_full", g, half))
                yield None
            if pair:
                self.arrive(("turn", 1 - g, w))
                yield None
        if n_u > 0:
            yield ("o_full", g), 0
            self.holds(("o", g), n_t - 1 if pair else 2 * (n_u - 1) + g)

    def piece(self, n_t, pair, valid_warps):
        rng = self.rng
        self.base = dict(self.done)
        self.copies, self.queue, self.running = [], [[], []], []
        self.mem = {k: v for k, v in self.mem.items() if not (isinstance(k[0], tuple) and k[0][0] == "go")}
        roles = [self.loader(kv, n_t) for kv in range(2)] + [self.products(g, n_t, pair) for g in range(2)]
        roles += [self.widener(kv, turn, which, n_t, pair) for kv in range(2) for turn in range(2) for which in range(2)]
        roles += [self.softmax(g, w, n_t, pair, w < valid_warps[g]) for g in range(2) for w in range(4)]
        waits = {r: None for r in roles}
        slow = {r: rng.random() ** 3 + 0.01 for r in roles}                     # some are much slower than others
        slow_product = [rng.random() ** 2 + 0.02 for _ in range(2)]
        idle = 0
        while waits or self.copies or any(self.queue):
            moved = False
            for r in rng.sample(list(waits), len(waits)):
                if rng.random() > slow[r]:
                    moved = True                                                # (it could go on, for all one knows)
                    continue
                w = waits[r]
                if w is not None and not (w() if callable(w) else self.passes(*w)):
                    continue
                moved, idle = True, 0
                try:
                    waits[r] = next(r)
                except StopIteration:
                    del waits[r]
            for copy in list(self.copies):                                      # in any order, some much later than others
                if rng.random() < copy[3]:
                    self.copies.remove(copy)
                    self.mem[copy[0]] = copy[1]
                    self.arrive(copy[2])
                    idle = 0
            for g in range(2):
                if self.queue[g] and rng.random() < slow_product[g]:
                    what, where, reads, writes, bars = self.queue[g][0]
                    for place, name in reads:
                        self.holds(place, name)
                    if (what, where) not in self.running:                       # begins; ends some time later
                        self.running.append((what, where))
                        continue
                    self.running.remove((what, where))
                    self.queue[g].pop(0)
                    for place, name in writes:
                        self.mem[place] = name
                    for bar, n in bars:
                        self.arrive(bar, n)
                    idle = 0
            idle += 1
            if idle > 20000:
                raise _Wrong(f"standstill: {[w for w in waits.values() if w is not None and not callable(w)]}")
        for b in self.done:
            self.odd[b] = (self.odd[b] + self.uses(b, n_t, pair, self.stages, self.full)) & 1
            if self.odd[b] != self.done[b] & 1:
                raise _Wrong(f"{b}: {self.done[b]} phases, taken for an {'odd' if self.odd[b] else 'even'} number")


def _play(seed, stages, full):
    rng = random.Random(seed)
    m = _Model(rng, stages, full)
    for _ in range(rng.randint(1, 5)):
        pair = rng.random() < 0.5
        valid = (4, rng.randint(1, 4)) if pair else (rng.randint(1, 4),) * 2
        m.piece(rng.choice((0, 1, 1, 2, 3, 5, 9, 14)), pair, valid)


def test_the_whole_kernels_model_finds_the_fault_of_too_few_barriers():
    found = 0
    for seed in range(40):
        try:
            _play(seed, 3, 3)
        except _Wrong:
            found += 1
    assert found > 10


@pytest.mark.parametrize("part", range(8))
def test_the_whole_kernel_in_any_order(part):
    for seed in range(1000 * part, 1000 * part + 25):
        _play(seed, *_constants())
