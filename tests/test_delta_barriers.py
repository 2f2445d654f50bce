"""The order in which the warps of the delta rule's tensor-core scan meet (csrc/delta_scan_tc.cu), played through on the CPU.

A wait asks for the parity of a barrier's phase alone: a warp that comes to it after the next phase has ended too waits for one that never ends.  So
whatever warp is late, and wherever, the others must not get two phases ahead of any wait of its.  Every warp is stopped before each of its steps in
turn, the others go on as far as they can, and then the stopped one's next wait is looked at."""
import pytest

NEED = {"empty_v": 8, "s": 8, "xp": 8, "wp": 8, "up": 8, "join": 8, "pair": 8, "out": 4, "scaled": 4}      # arrivals that end a phase; others: one


def roles(units):
    """[(name, [(wait or arrive, barrier, phase)])] of a CTA's units: (outputs, stored state, chunks, those that are looked at, and then taken token by
    token)."""
    chunks = [(outputs, stored or i > 0, i == 0, i == n - 1, i in looked, i in alone) for outputs, stored, n, looked, alone in units for i in range(n)]
    two = lambda bar, n: (f"{bar}{n & 1}", n >> 1)  # noqa: E731
    copies, products, values, store = [], [], [], []
    y, state = [], []
    o = om = m = u = met = 0
    for n, (outputs, live, first, last, looked, alone) in enumerate(chunks):
        wait, arrive = lambda to: lambda bar, k: to.append(("wait", bar, k)), lambda to: lambda bar: to.append(("arrive", bar, None))
        # the copies
        if n >= 2:
            wait(copies)(*two("empty", n - 2))
        arrive(copies)(two("full", n)[0])
        # the products
        w, a = wait(products), arrive(products)
        w(*two("full", n))
        if live:
            w("s0", m), w("s1", m), a("x")
        w("xp", n), a("u")
        if outputs and o:
            w("out", o - 1)
        if live and outputs:
            a("ask")
        w("wp", n), a("prod")
        if outputs:
            w(*two("up", o))
            if live:
                w("scaled", om)
            a("y")
        a(two("empty", n)[0])
        # the values, a copy ahead
        w, a = wait(values), arrive(values)
        for c in ([0, 1] if n == 0 else [n + 1]):
            if c < len(chunks):
                if c >= 2:
                    w(*two("empty_v", c - 2))
                a(two("raw", c)[0])
        w(*two("raw", n)), a(two("full_v", n)[0])
        # the state
        w, a = wait(state), arrive(state)
        if first:
            w(*two("full_v", n)), a(two("empty_v", n)[0]), a("join"), w("join", u)
            u += 1
            if live:
                a("s0"), a("s1")
        w(*two("full", n))
        if looked or alone:
            if o:
                w(*two("out_free", o - 1))
            for _ in range(4 if alone else 1):
                a("pair"), w("pair", met)
                met += 1
        if not last and not alone:
            w(*two("full_v", n + 1)), a(two("empty_v", n + 1)[0])
        if live:
            w("x", m)
        a("xp"), w("u", n), a("wp")
        if outputs:
            a(two("up", o)[0])
        if not last and alone:
            w(*two("full_v", n + 1))
        w("prod", n)
        if not last:
            a("s0"), a("s1")
        if not last and alone:
            w(*two("full_v", n + 1)), a(two("empty_v", n + 1)[0])
        # the outputs
        if outputs:
            w, a = wait(y), arrive(y)
            if live:
                w(*two("full", n)), w("ask", om), a("scaled")
            w(*two("up", o)), w("y", o)
            if o:
                w(*two("out_free", o - 1))
            a("out")
            wait(store)("out", o), arrive(store)(two("out_free", o)[0])
            o += 1
            om += live
        m += live
    return [("copies", copies), ("products", products), ("values", values), ("store", store)] + [(f"state {i}", state) for i in range(8)] + [(f"y {i}", y) for i in range(4)]


class Play:
    def __init__(self, units):
        self.roles, self.done, self.count = roles(units), {}, {}
        self.at = [0] * len(self.roles)

    def ready(self, r):
        kind, bar, k = self.roles[r][1][self.at[r]]
        return kind == "arrive" or (self.done.get(bar, 0) & 1) != (k & 1)

    def run(self, r, end):
        """Warp r up to its step `end`, as far as it gets."""
        start, ops = self.at[r], self.roles[r][1]
        while self.at[r] < min(end, len(ops)) and self.ready(r):
            kind, bar, k = ops[self.at[r]]
            if kind == "arrive":
                self.count[bar] = self.count.get(bar, 0) + 1
                if self.count[bar] == NEED.get(bar.rstrip("01"), 1):
                    self.count[bar], self.done[bar] = 0, self.done.get(bar, 0) + 1
            else:
                assert self.done[bar] == k + 1, (self.roles[r][0], bar, k, self.done[bar])
            self.at[r] += 1
        return self.at[r] > start

    def all(self, stopped=None, end=0):
        while any([self.run(r, end if r == stopped else 1 << 30) for r in range(len(self.roles))]):
            pass


# whole sequences from zeros and from stored states, of one chunk and more; the first pass over segments, without outputs (a CTA's units have them all, or
# none has)
UNITS = [[(True, False, 1, (), ())], [(True, False, 2, (), (0,))], [(True, True, 5, (2, 3), (0, 1, 4))],
         [(True, False, 4, (), (2,)), (True, True, 1, (), (0,)), (True, False, 1, (0,), ()), (True, True, 3, (1,), ())],
         [(False, False, 4, (2,), (1, 3)), (False, True, 3, (0,), ())]]


@pytest.mark.parametrize("units", UNITS)
def test_no_warp_gets_two_phases_ahead_of_a_wait(units):
    whole = Play(units)
    whole.all()
    assert whole.at == [len(ops) for _, ops in whole.roles]
    for r in [0, 1, 2, 3, 4, 12]:                        # (one of the state's warps and one of Y's stand for all)
        name, ops = whole.roles[r]
        for i in range(len(ops)):
            p = Play(units)
            p.all(r, i)
            assert p.at[r] == i
            kind, bar, k = ops[i]
            if kind == "wait":
                assert p.done.get(bar, 0) <= k + 1, (name, i, bar, k)
            p.all()
            assert p.at == whole.at
