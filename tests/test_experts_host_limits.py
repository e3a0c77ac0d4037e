"""What the operators of a Dense Part made of experts check on the host before anything runs, where lists and devices go wrong."""
import itertools
import random

import pytest

from paper_1806_03925_amd import experts


@pytest.mark.parametrize("src,dst,shared", [
    ([(0, 8), (8, 8)], [(0, 8), (8, 8)], False),            # in place, neighbours
    ([(0, 8), (0, 8)], [(0, 8), (0, 8)], True),             # a tensor twice, in place
    ([(0, 8), (0, 8)], [(64, 8), (72, 8)], False),          # a tensor twice, scaled into two others
    ([(0, 8), (16, 8)], [(64, 8), (64, 8)], True),          # two results in one place
    ([(0, 8), (16, 8)], [(64, 8), (71, 8)], True),
    ([(0, 8), (16, 8)], [(16, 8), (0, 8)], True),           # in one another's place
    ([(0, 8), (16, 8)], [(64, 8), (0, 8)], True),           # one result in another's source
    ([(0, 8)], [(4, 8)], True),                             # shifted against its own source
    ([(0, 0), (0, 8), (4, 0)], [(0, 0), (0, 8), (4, 0)], False),   # tensors without elements are nowhere
    ([], [], False)])
def test_memory_that_gradients_share(src, dst, shared):
    assert experts._share_memory(src, dst) is shared


def test_memory_that_gradients_share_against_every_pair():
    rng = random.Random(5)
    seen = set()
    for _ in range(3000):
        n = rng.randint(1, 5)
        size = [rng.randint(0, 4) for _ in range(n)]
        src = [(rng.randint(0, 30), s) for s in size]
        dst = [a if rng.random() < 0.6 else (rng.randint(0, 60), a[1]) for a in src]
        meet = lambda a, b: set(range(a[0], sum(a))) & set(range(b[0], sum(b)))
        want = any(meet(a, b) for a, b in itertools.combinations(dst, 2))
        want = want or any(meet(s, d) and not (i == j and s == d) for i, s in enumerate(src) for j, d in enumerate(dst))
        assert experts._share_memory(src, dst) is bool(want), (src, dst)
        seen.add(bool(want))
    assert seen == {True, False}
