"""How the warps of the prompts' kernel over an 8-bit cache wait for one another, as a model on the CPU.

Every warp of a block is a generator that yields its waits; the tensor core is one more, which carries out what the products'
warp has issued, in order, later.  Schedules are random, some warps starved.  Checked is what each warp finds where it reads
(items, stages of K and V, scales, scores, weights, outputs, NaN keys) and that nothing is overwritten that somebody still
reads.  Waits may also give up, as the kernel's do after about a second: the results are then worth nothing, but every warp has
to reach the block's end, and no product may be on its way when tensor memory is given back."""
import pathlib
import random
import re

import pytest

SOURCE = pathlib.Path(__file__).parents[1] / "paper_2608_12703_gb300" / "csrc" / "paged8_prompt.cu"


class Wrong(Exception):
    pass


class Bar:
    """An mbarrier: `count` arrivals end a phase."""

    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1

    def passed(self, parity):   # of the phase of that parity, the current or the one before: no more is known
        return self.done & 1 != parity


class Block:
    """`items`: key tiles (n0, n1) of the two row tiles.  `faults`: ways in which the protocol is made wrong."""

    def __init__(self, seed, items, once, late=0.0, faults=()):
        self.rng, self.items, self.once, self.faults = random.Random(seed), items, once, set(faults)
        self.late, self.given_up = late, False     # chance that a wait gives up
        new = lambda n, count: [Bar(count) for _ in range(n)]
        self.q_full, self.k_full, self.v_full = new(2, 4), new(2, 3), new(2, 3)
        self.k_free, self.v_free = new(2, 1), new(2, 1)
        self.pv_done = [new(4, 1), new(4, 1)]
        self.s_full, self.p_full, self.sc_full = new(2, 1), new(2, 4), new(8, 2)
        self.item_full, self.begun, self.ended, self.drained = new(4, 1), new(4, 1), new(4, 14), Bar(1)
        self.slots, self.nan = [None] * 4, [None] * 4
        self.stage = {"k": [None, None], "v": [None, None]}
        self.written = {"k": [set(), set()], "v": [set(), set()]}
        self.scales = [{}, {}, {}, {}, {}, {}, {}, {}]
        self.q, self.s, self.p, self.o = [{}, {}], [None, None], [{}, {}], [None, None]
        self.used = [None, None]        # weights of a buffer that have been multiplied
        self.reads_o = [0, 0]           # weighing warps of a row tile that have yet to read its outputs
        self.queue, self.seen, self.out = [], {}, {}
        self.named, self.at_named = 0, 0
        self.lag = 2 if once else 1
        self.warps = {f"w{x}{w}": self.weigh(x, w) for x in (0, 1) for w in range(4)}
        self.warps |= {f"k{w}": self.convert("k", w) for w in range(3)} | {f"v{w}": self.convert("v", w) for w in range(3)}
        self.warps["p"] = self.products()

    def check(self, ok, what):
        if not ok and not self.given_up:
            raise Wrong(what)

    def waits_on(self, what):   # products on their way that use `what`
        return any(what in op[1] for op in self.queue)

    # ---------------------------------------------------------------- the schedule
    def run(self):
        rng, ready = self.rng, dict.fromkeys(self.warps)
        weight = {name: rng.choice((0.02, 0.3, 1, 1, 1)) for name in [*self.warps, "core"]}
        gave_up = dict.fromkeys(self.warps, False)
        for _ in range(2_000_000):
            if not ready:
                if self.queue:
                    raise Wrong("products on their way at the end")
                return
            able = [n for n, w in ready.items() if w is None or gave_up[n] and w[0] != "all" or self.passed(w)] + (["core"] if self.queue else [])
            stuck = not able
            if stuck:      # time passes: a wait with a limit gives up
                able = [n for n, w in ready.items() if w[0] != "all"]
                if not able or not self.late:
                    raise Wrong(f"nothing goes on: {ready}")
            name = rng.choices(able, [weight[n] for n in able])[0]
            if name == "core":
                self.carry_out()
                continue
            w = ready[name]
            if w is not None and w[0] != "all" and (stuck or self.late and rng.random() < self.late):
                gave_up[name] = self.given_up = True
            try:
                ready[name] = self.warps[name].send(None if w is None else gave_up[name])
            except StopIteration:
                del ready[name]
        raise Wrong("no end")

    def passed(self, w):
        return self.named >= w[1] if w[0] == "all" else w[0].passed(w[1])

    def carry_out(self):
        self.queue.pop(0)[2]()

    # ---------------------------------------------------------------- items
    def fetch(self, k):
        late = False
        if k >= 4:
            late = yield self.ended[k & 3], (k >> 2) - 1 & 1
        self.slots[k & 3] = k if k < len(self.items) else -1
        if "named barrier" not in self.faults:
            self.nan[k & 3] = k
        self.item_full[k & 3].arrive()
        return late

    def take(self, k):
        late = yield self.item_full[k & 3], k >> 2 & 1
        i = -1 if late else self.slots[k & 3]
        self.check(i == k or i == -1 and k >= len(self.items), f"item {k}: {i}")
        return i

    # ---------------------------------------------------------------- the warps
    def weigh(self, x, w):
        tiles = pairs = steps = 0
        n0 = n1 = nx = 0
        k, idle = -1, False
        while True:
            if nx > 0 and idle and "no begun" not in self.faults:
                yield self.begun[k & 3], k >> 2 & 1
            idle = nx == 0
            nxt = yield from self.take(k + 1)
            for j in range(nx):
                pair, tile = pairs + min(j, n0) + min(j, n1) + (x == 1 and j < n0), tiles + j
                buf = pair % 2
                yield self.sc_full[tile & 7], tile >> 3 & 1
                yield self.s_full[buf], pair // 2 & 1
                yield None
                self.check(self.scales[tile & 7].get("k") == self.scales[tile & 7].get("v") == (k, j), "scales")
                self.check(self.s[buf] == (k, x, j), f"scores {self.s[buf]} for {(k, x, j)}")
                moves = j > 0 and self.rng.random() < 0.3

                def added():
                    yield self.pv_done[x][(steps + j - 1) & 3], (steps + j - 1) >> 2 & 1
                if j > 0 and (self.once and "weights early" not in self.faults or moves):
                    yield from added()
                if moves:
                    self.check(not self.waits_on(("o", x)) and self.o[x] == (k, j), "outputs moved while they are added to")
                if self.once:
                    self.check(not self.waits_on(("p", buf)), "weights over weights in use")
                self.p[buf][w] = (k, x, j)
                yield None
                self.seen.setdefault((k, j), set()).add((x, w))
                self.p_full[buf].arrive()
            pairs, tiles, steps = pairs + n0 + n1, tiles + max(n0, n1), steps + nx
            was, k, was_nx = k, k + 1, nx
            n0, n1 = self.items[nxt] if nxt >= 0 else (0, 0)
            nx = n1 if x else n0
            if nx > 0:
                self.check(not self.waits_on(("q", x)), "q over a q in use")
                self.q[x][w] = k
                self.q_full[x].arrive()
            if was >= 0:
                if was_nx > 0:
                    yield self.pv_done[x][(steps - 1) & 3], (steps - 1) >> 2 & 1
                    yield None
                    self.check(self.o[x] == (was, was_nx) and not self.waits_on(("o", x)), f"outputs {self.o[x]} of {was}")
                    self.reads_o[x] -= 1
                self.check(self.nan[was & 3] == was, f"NaN keys of {self.nan[was & 3]} for {was}")
                self.out.setdefault(was, set()).add((x, w))
                self.ended[was & 3].arrive()
            if nxt < 0:
                return

    def convert(self, what, w):
        full, free = (self.k_full, self.k_free) if what == "k" else (self.v_full, self.v_free)
        first, k, tile, gave_up, rounds = what == "k" and w == 0, -1, 0, False, 0
        i = 0
        while True:
            k += 1
            if first:
                if k == 0:
                    yield from self.fetch(0)
                yield from self.fetch(k + 1)
            i = yield from self.take(k)
            if i < 0:
                return
            for j in range(max(self.items[i])):
                st = tile & 1
                if w == 0:
                    old = self.scales[tile & 7].get(what)
                    if old is not None:
                        n = self.items[old[0]]
                        want = {(x, v) for x in (0, 1) for v in range(4) if old[1] < n[x]}
                        self.check(want <= self.seen.get(old, set()), "scales over scales in use")
                    self.scales[tile & 7][what] = (i, j)
                    yield None
                    self.sc_full[tile & 7].arrive()
                if what == "v":
                    if j == 0 and "named barrier" in self.faults:
                        self.nan[k & 3], rounds = k, rounds + 1
                        self.at_named += 1
                        self.named += self.at_named % 3 == 0
                        yield "all", rounds
                    self.check(self.nan[k & 3] == k, "NaN keys of another item")
                if tile >= 2:
                    yield free[st], (tile >> 1) - 1 & 1
                self.check(not self.waits_on((what, st)), "a stage over one in use")
                self.stage[what][st] = (i, j)
                self.written[what][st].add((i, j, w))
                yield None
                full[st].arrive()
                tile += 1
            if not first:
                self.ended[k & 3].arrive()

    def products(self):
        pairs = tiles = 0
        q_of, pv_of = [0, 0], [0, 0]
        k = 0

        def issue(kind, uses, act):
            self.queue.append((kind, uses, act))

        def commit(bar):
            issue("commit", (), bar.arrive)
        while True:
            i_item = yield from self.take(k)
            if i_item < 0:
                break
            n0, n1 = self.items[i_item]
            n = n0 + n1
            self.begun[k & 3].arrive()

            def place(i):
                return (0, i) if n1 == 0 else (i & 1 if i < 2 * n0 else 1, i >> 1)
            for i in range(n + self.lag):
                o, o_buf = i - self.lag, (pairs + i - self.lag) & 1
                if self.once and o >= 0:
                    yield self.p_full[o_buf], (pairs + o) >> 1 & 1
                if i < n:
                    (x, j), buf = place(i), (pairs + i) & 1
                    st = tiles + j & 1
                    if j == 0:
                        q_of[x] += 1
                        yield self.q_full[x], q_of[x] - 1 & 1
                    yield self.k_full[st], tiles + j >> 1 & 1

                    def scores(x=x, j=j, st=st, buf=buf, k=k):
                        self.check(self.stage["k"][st] == (k, j) and all((k, j, w) in self.written["k"][st] for w in range(3)), "keys")
                        self.check(all(self.q[x].get(w) == k for w in range(4)), "q")
                        was = self.s[buf]
                        if was:     # scores that have been weighed, and, where weights take their place, multiplied
                            self.check({(was[1], w) for w in range(4)} <= self.seen.get((was[0], was[2]), set()), "scores over scores")
                            self.check(self.once or self.used[buf] == was, "scores over weights")
                        self.s[buf] = (k, x, j)
                    issue("scores", (("k", st), ("q", x), ("s", buf)), scores)
                    commit(self.s_full[buf])
                    if x == 1 or j >= n1:
                        commit(self.k_free[st])
                    yield None
                if o >= 0:
                    x, j = place(o)
                    st = tiles + j & 1
                    yield self.v_full[st], tiles + j >> 1 & 1
                    if not self.once:
                        yield self.p_full[o_buf], (pairs + o) >> 1 & 1

                    def outputs(x=x, j=j, st=st, buf=o_buf, k=k):
                        self.check(self.stage["v"][st] == (k, j) and all((k, j, w) in self.written["v"][st] for w in range(3)), "values")
                        self.check(all(self.p[buf].get(w) == (k, x, j) for w in range(4)), "weights")
                        if j == 0:
                            self.check(self.reads_o[x] == 0, "outputs over outputs that are still read")
                            self.reads_o[x] = 4
                        else:
                            self.check(self.o[x] == (k, j), "outputs")
                        self.o[x], self.used[buf] = (k, j + 1), (k, x, j)
                    issue("outputs", (("v", st), ("p", o_buf), ("o", x)), outputs)
                    pv_of[x] += 1
                    commit(self.pv_done[x][(pv_of[x] - 1) & 3])
                    if x == 1 or j >= n1:
                        commit(self.v_free[st])
                    yield None
            pairs, tiles = pairs + n, tiles + max(n0, n1)
            self.ended[k & 3].arrive()
            k += 1
        if "not drained" not in self.faults:
            commit(self.drained)
            late = yield self.drained, 0
            if late:      # the kernel's last wait begins with a limit of its own; the core needs far less
                while self.queue:
                    self.carry_out()


def some_items(rng):
    items = []
    for _ in range(rng.randint(1, 12)):
        n0 = rng.choice((1, 1, 2, 3, 5, 9))
        items.append((n0, rng.choice((0, 0, n0, n0 + 1))))
    return items


def runs(n, **kw):
    for seed in range(n):
        yield Block(seed, some_items(random.Random(seed)), once=seed % 2 == 0, **kw)


def test_all_items_come_out_right():
    for block in runs(400):
        block.run()
        assert len(block.out) == len(block.items) and all(len(v) == 8 for v in block.out.values())


@pytest.mark.parametrize("late", [0.0005, 0.01])
def test_warps_whose_waits_give_up_leave_no_one_behind(late):
    gave_up = 0
    for block in runs(400, late=late):
        block.run()
        gave_up += block.given_up
    assert gave_up > 50


@pytest.mark.parametrize("fault,late", [("named barrier", 0.002), ("not drained", 0.01), ("no begun", 0.0), ("weights early", 0.0)])
def test_the_model_sees_what_would_be_wrong(fault, late):
    """A barrier without a limit among warps of which one has left; products on their way at the end; a row tile that sat out an
    item and takes an older phase for its own; weights over those that are being multiplied."""
    found = 0
    for block in runs(400, late=late, faults=[fault]):
        try:
            block.run()
        except Wrong:
            found += 1
    assert found > 0


def test_the_kernel_is_the_one_of_the_model():
    """Barriers, their counts, and that no warp waits without a limit between the block's first and last barrier."""
    text = SOURCE.read_text()
    bars = re.search(r"struct Prompt8Bars \{[^\n]*\n(.*?)\n\};", text, re.S).group(1)
    block = Block(0, [(1, 1)], True)
    sizes = {n: int(c or 1) for n, c in re.findall(r"(\w+)(?:\[(\d+)\])?(?:\[\d+\])?(?=[,;])", bars)}
    counts = {n: int(eval(c)) for n, c in re.findall(r"mbar_init\(&bars\.(\w+)(?:\[\w\])*, ([\d +]+)\)", text)}
    assert sizes.keys() == counts.keys()
    for name, count in counts.items():
        got = getattr(block, name)
        got = got if isinstance(got, list) else [got]
        assert len(got) <= sizes[name], name
        assert all(b.count == count for g in got for b in (g if isinstance(g, list) else [g])), name
    assert "constexpr int LAG = ONCE ? 2 : 1;" in text and "NS = 2;" in text
    roles = text[text.index("if (warp < 8) asm volatile"):text.index("if (warp == 14) tmem_dealloc")]
    roles = roles[:roles.rindex("__syncthreads")]
    assert not re.search(r"__syncthreads|bar\.sync|barrier\.|mbar_wait\(|while \(!?mbar", roles)
