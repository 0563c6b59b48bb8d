"""Which results of a reordering overlap something else of the call, by addresses alone: the
helper refuses those, since rows would be written while others are read. Without a GPU; the
reference marks every byte."""
import itertools
import random

import pytest

from paper_2609_38477_amd.beam import _races


def bytes_of(region):
    at, row, rows, step, outer, inner, _ = region
    return {at + r * row + o * step + i for r in range(rows) for o in range(outer) for i in range(inner)}


def by_marks(regions) -> bool:
    marks = [bytes_of(r) for r in regions]
    return any((a[6] or b[6]) and not s.isdisjoint(t)
               for (a, s), (b, t) in itertools.combinations(zip(regions, marks), 2))


def test_by_hand():
    a = (4096, 100, 4, 0, 1, 100, True)                    # four dense rows of 100 bytes
    assert not _races([a])
    assert not _races([a, (4496, 100, 4, 0, 1, 100, True)])          # right after it
    assert _races([a, (4495, 100, 4, 0, 1, 100, False)])             # its last byte
    assert _races([a, (4200, 0, 1, 0, 1, 8, False)])                 # the parents inside a result
    read = (4096, 100, 4, 0, 1, 100, False)
    assert _races([a, read]) and not _races([read, read])
    # a row that another tensor's rows lie in, one byte too long or not
    assert not _races([(0, 64, 8, 0, 1, 24, True), (24, 64, 8, 0, 1, 40, True)])
    assert _races([(0, 64, 8, 0, 1, 25, True), (24, 64, 8, 0, 1, 40, True)])
    assert _races([(0, 64, 8, 0, 1, 24, True), (24, 64, 8, 0, 1, 41, True)])
    assert not _races([(0, 64, 8, 0, 1, 24, True), (24 + 64 * 3, 64, 8, 0, 1, 40, True)])
    # one state twice, moved in place for one of its results: the other reads what is written
    assert _races([a, read, (9000, 100, 4, 0, 1, 100, True)])


@pytest.mark.parametrize("layers,rows,heads,used,width", [(32, 16, 8, 100, 64), (5, 1, 3, 7, 2)])
def test_layers_inside_one_tensor(layers, rows, heads, used, width):
    # [rows][layer][key or value][heads][room][width], the used part of each moved in place
    room = used + 3
    size = heads * room * width
    row = 2 * layers * size
    regions = [((1 << 20) + k * size, row, rows, room * width, heads, used * width, True) for k in range(2 * layers)]
    parents = ((1 << 20) + rows * row, 0, 1, 0, 1, 8 * rows, False)
    assert not _races(regions + [parents])
    far = [(r[0] + 3 * rows * row + 17, *r[1:6], False) for r in regions]     # and read from another one
    assert not _races(regions + far)
    near = list(regions)
    near[-1] = (near[-1][0] - (3 * width + 1), *near[-1][1:])
    assert _races(near)
    # [rows][heads][layer][room][width]
    piece = room * width
    step = layers * piece
    inside = [((1 << 20) + k * piece, heads * step, rows, step, heads, used * width, True) for k in range(layers)]
    assert not _races(inside)
    inside[0] = (*inside[0][:5], piece + 1, True)
    assert _races(inside)


@pytest.mark.parametrize("seed", range(8))
def test_random_layouts(seed):
    rng = random.Random(seed)
    seen = {True: 0, False: 0}
    for _ in range(1500):
        n, regions = rng.randint(2, 4), []
        strides = [rng.choice((0, 6, 8, 12, 24, 30, 48, 60)) for _ in range(3)]
        for _ in range(n):
            regions.append((rng.randint(0, 150), rng.choice(strides), rng.randint(1, 4), rng.choice(strides),
                            rng.randint(1, 4), rng.randint(1, 7), rng.random() < 0.6))
        want = by_marks(regions)
        assert _races(regions) == want, regions
        seen[want] += 1
    assert min(seen.values()) > 100
