"""Which outputs a table of gradients may have, by their places alone (no GPU): a clipping reads and
writes all of them at once, so none may meet another entry's output or gradient."""
import random

import pytest

from paper_2607_08782_amd import moe


@pytest.mark.parametrize("reads,writes,nbytes,apart", [
    ([], [], [], True),
    ([64], [64], [16], True),                        # in place
    ([64, 80], [64, 80], [16, 16], True),            # side by side
    ([64, 64], [256, 512], [16, 16], True),          # one gradient twice, outputs apart
    ([64, 72], [256, 512], [16, 16], True),          # gradients that overlap
    ([64, 64], [64, 64], [16, 16], False),           # one output twice
    ([64, 64], [256, 256], [16, 16], False),
    ([64, 72], [64, 72], [16, 16], False),           # views that overlap, in place
    ([64, 256], [512, 520], [64, 4], False),         # an output inside another
    ([64, 256], [520, 512], [4, 64], False),
    ([64, 256], [256, 64], [16, 16], False),         # swapped
    ([64, 256], [512, 64], [16, 16], False),         # one over another's gradient
    ([64, 256], [512, 60], [16, 8], False),
    ([64, 64], [64, 256], [16, 16], False),          # read by one, written by another
    ([64], [72], [16], False),                       # over part of its own
    ([64], [56], [16], False),
    ([64], [80], [16], True),
    ([64, 64, 70], [64, 64, 70], [0, 16, 0], True),  # nothing to read or write
])
def test_outputs_apart(reads, writes, nbytes, apart):
    assert moe._outputs_apart(reads, writes, nbytes) is apart
    assert moe._outputs_apart(reads[::-1], writes[::-1], nbytes[::-1]) is apart


def test_outputs_apart_against_bytes():
    """Against the definition, byte by byte."""
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(3000):
        n = rng.randint(1, 4)
        sizes = [rng.choice((0, 1, 2, 3, 5)) for _ in range(n)]
        reads = [rng.randrange(20) for _ in range(n)]
        writes = [r if rng.random() < 0.5 else rng.randrange(20) for r in reads]
        cells = lambda at, size: set(range(at, at + size))
        want = True
        for i in range(n):
            out = cells(writes[i], sizes[i])
            for j in range(n):
                if i != j and out & cells(writes[j], sizes[j]):
                    want = False
                if out & cells(reads[j], sizes[j]) and not (i == j and reads[i] == writes[i]):
                    want = False
        assert moe._outputs_apart(reads, writes, sizes) is want, (reads, writes, sizes)
        seen[want] += 1
    assert min(seen) > 300
