"""The tickets of a counter in memory that may hold anything (draw_any in csrc/device_utils.h), its steps written out for the CPU: whatever was there and
however the workgroups' atomics follow one another, each draws, no ticket is drawn twice, and drawing ends."""
import itertools
import os
import random

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TAG, LOW = 0x6A09E667, (1 << 32) - 1


def drawing(memory, tickets):
    """One workgroup; a step of the generator is one atomic."""
    def counts(word):
        return word >> 32 == TAG and word & LOW < tickets
    while True:
        seen = memory[0]
        memory[0] = (seen + 1) % (1 << 64)
        yield
        if counts(seen):
            return seen & LOW
        seen = (seen + 1) % (1 << 64)
        while not counts(seen):
            was = memory[0]
            if was == seen:
                memory[0] = TAG << 32 | 1
            yield
            if was == seen:
                return 0
            seen = was


def run(start, tickets, order):
    """The tickets, by an order of the workgroups' atomics (an iterator of numbers, taken modulo those that still draw)."""
    memory, drawn = [start], {}
    going = {w: drawing(memory, tickets) for w in range(tickets)}
    for step in range(1000 * tickets):
        if not going:
            break
        w = sorted(going)[next(order) % len(going)]
        try:
            next(going[w])
        except StopIteration as done:
            drawn[w] = done.value
            del going[w]
    assert not going, "drawing did not end"
    assert sorted(drawn.values()) == list(range(tickets)), (hex(start), drawn)
    assert memory[0] == TAG << 32 | tickets
    return max(drawn, key=drawn.get)


STARTS = [0, 1, 2, 3, LOW, LOW + 1, (1 << 64) - 1, (1 << 64) - 2, TAG << 32, (TAG << 32) + 3, (TAG << 32) + LOW, (TAG << 32) - 2, 0x3F8000003F800000]


def test_every_order_of_a_few():
    for start in STARTS:
        for tickets in (1, 2, 3):
            if start >> 32 == TAG and 0 < start & LOW < tickets:
                continue                                               # looks like a count
            for order in itertools.product(range(tickets), repeat=8 if tickets == 3 else 6):
                run(start, tickets, itertools.chain(order, itertools.cycle(range(tickets))))


def test_random_orders_of_many():
    rng = random.Random(1)
    for _ in range(300):
        start, tickets = rng.choice(STARTS + [rng.getrandbits(64)]), rng.choice((4, 17, 128))
        if not (start >> 32 == TAG and 0 < start & LOW < tickets):
            run(start, tickets, iter(lambda: rng.getrandbits(16), None))


def test_the_tag_is_the_kernels():
    text = open(os.path.join(ROOT, "paper_2106_05203_amd", "csrc", "device_utils.h")).read()
    assert "kCounts = 0x6A09E667u" in text
