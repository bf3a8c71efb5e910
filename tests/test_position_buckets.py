"""position_buckets: borders of buckets against their definition in whole numbers, large distances, and bounds that are told at once."""
import random
import time

import pytest

import paper_1911_00472_amd as pkg


def side_of(e, c, f, reach):
    """The bucket of every distance: from e on e + j for the last j below c with x^c >= e^(c - j) f^j."""
    side, j = [], 0
    for x in range(reach + 1):
        while j + 1 < c and x ** c >= e ** (c - j - 1) * f ** (j + 1):
            j += 1
        side.append(x if x < e else e + j if c else e - 1)
    return side


def test_borders_are_those_of_the_definition():
    rng = random.Random(1)
    cases = [(1, 1, 2), (1, 24, 2 ** 10), (8, 8, 128), (16, 16, 128), (3, 7, 4), (1, 100, 4), (5, 40, 3125), (2, 30, 2 ** 11), (7, 50, 343), (6, 5, 46656), (10, 3, 1000), (1, 25, 2 ** 12), (9, 48, 729)]
    cases += [(e, c, e + rng.randrange(1, 400)) for e in range(1, 20) for c in (1, 2, 3, 5, 8, 12, 27, 64)]
    for e, c, f in cases:
        m, n = pkg.position_buckets(e, c, f, device="cpu")
        assert n == 2 * (e + c) - 1 and m.shape == (1, 2 * f + 1)
        side = side_of(e, c, f, f)
        assert m[0, f:].tolist() == [e + c - 1 + v for v in side] and m[0, :f + 1].tolist() == [e + c - 1 - v for v in side[::-1]], (e, c, f)
        m, n = pkg.position_buckets((e, 2), (c, 0), (f, 0), one_sided=True, device="cpu")
        assert n == (e + c) * 2 and m[0, :f + 1].flip(0).tolist() == [2 * v for v in side] and not m[0, f:].any(), (e, c, f)


@pytest.mark.parametrize("e,c", [(8, 15), (3, 1), (100, 5000), (2 ** 20, 2 ** 20), (1, 4000000)])
def test_the_largest_distances(e, c):
    begin = time.monotonic()
    m, n = pkg.position_buckets(e, c, 2 ** 24, device="cpu")
    assert time.monotonic() - begin < 30
    assert n == 2 * (e + c) - 1 and m.shape == (1, 2 ** 25 + 1)
    row = m[0, 2 ** 24:]
    assert int(row[0]) == e + c - 1 and int(row[-1]) == n - 1 and bool((row[1:] >= row[:-1]).all())
    if c < 100:                                                # a border, a whole number as it is defined
        j = c // 2
        x = next(x for x in range(int(e * (2 ** 24 / e) ** (j / c)) - 1, 2 ** 24) if x ** c >= e ** (c - j) * 2 ** (24 * j))
        assert int(row[x]) == e + c - 1 + e + j and (j == 0 or int(row[x - 1]) == e + c - 1 + e + j - 1)


@pytest.mark.parametrize("how", [(8, 8, 2 ** 24 + 1), (8, 8, 2 ** 40), (8, 8, 10 ** 30), (2 ** 24 + 2, 0, 0), (10 ** 12,), (1, 2 ** 24, 5), (8, 10 ** 15, 100), ((4000, 4000), (1000, 1000), (5000, 9000))])
def test_what_is_out_of_range_is_told_at_once(how):
    begin = time.monotonic()
    with pytest.raises(ValueError):
        pkg.position_buckets(*how, device="cpu")
    assert time.monotonic() - begin < 1
