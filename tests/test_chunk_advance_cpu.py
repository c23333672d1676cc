"""advance() by chunks whose bounds lie outside the packed rows: what append() takes, which cuts every
bound to the rows."""
import pytest
import torch

from test_chunk_calls_cpu import _Lens


def _taken(cu, total, counts, lens, max_context):
    """Tokens of every place that append() takes, from its description."""
    n = []
    for s, a in enumerate(lens):
        b = min(max(cu[s], 0), total)
        e = min(max(cu[s + 1], b), total)
        x = e - b if counts is None else max(0, min(e - b, counts[s]))
        n.append(min(x, max_context - a) if 0 <= a < max_context else 0)
    return n


CASES = [
    ([-5, 60, 124, 1 << 30], 224), ([-9, 40, 43, 1 << 30], 173), ([0, 10, 20, 30], 25), ([3, 3, 40, 41], 30),
    ([-(1 << 31), 5, 6, 2 ** 31 - 1], 7), ([-(1 << 31), -7, 2 ** 31 - 1, 2 ** 31 - 1], 9), ([40, 50, 60, 70], 30),
    ([0, 0, 0, 0], 12),
]


@pytest.mark.parametrize("cu,total", CASES, ids=lambda x: str(x))
@pytest.mark.parametrize("counts", [None, [1, 0, 7], [2 ** 31 - 1, -(1 << 31), 40]], ids=str)
def test_bounds_outside_the_rows(cu, total, counts):
    lens = [10, 0, 90]
    c = _Lens(lens, 300)
    c.advance(torch.tensor(cu, dtype=torch.int32), None if counts is None else torch.tensor(counts, dtype=torch.int32),
              total_tokens=total)
    assert c.lens.tolist() == [a + n for a, n in zip(lens, _taken(cu, total, counts, lens, 300))]
    assert c.lens.dtype is torch.int32


def test_bounds_below_zero_are_zero_without_the_rows():
    c = _Lens([10, 0, 90], 300)
    c.advance(torch.tensor([-5, 60, -(1 << 31), 70], dtype=torch.int32))
    assert c.lens.tolist() == [70, 0, 160]


def test_rows_and_room():
    lens = [299, -1, 300, 5, -(1 << 31)]
    c = _Lens(lens, 300)
    cu = [-1, 50, 60, 70, 80, 1 << 30]
    c.advance(torch.tensor(cu, dtype=torch.int32), total_tokens=75)
    assert c.lens.tolist() == [a + n for a, n in zip(lens, _taken(cu, 75, None, lens, 300))]


@pytest.mark.parametrize("cu,counts", [
    ([0, 5], None), ([0, 1, 2], None), ([0, 1, 2, 3, 4], None), ([0, 1, 2, 3], [1]), ([0, 1, 2, 3], [1, 1]),
    ([0, 1, 2, 3], [[1, 1, 1]]), ([[0, 1, 2, 3]], None), ([0.0, 1.0, 2.0, 3.0], None), ([0, 1, 2, 3], [True] * 3),
], ids=str)
def test_refusals(cu, counts):
    """As append() refuses them; broadcast, they would move every place."""
    c = _Lens([10, 0, 90], 300)
    x = torch.tensor(cu)
    x = x if x.is_floating_point() else x.to(torch.int32)
    y = None if counts is None else torch.tensor(counts)
    y = y if y is None or y.dtype is torch.bool else y.to(torch.int32)
    with pytest.raises(ValueError):
        c.advance(x, y)
    with pytest.raises(ValueError):
        c.advance(torch.arange(4), None)       # int64
    assert c.lens.tolist() == [10, 0, 90]


def test_counts_without_bounds_are_refused():
    c = _Lens([10, 0, 90], 300)
    for kw in (dict(counts=torch.tensor([1, 1, 1], dtype=torch.int32)), dict(total_tokens=3)):
        with pytest.raises(ValueError):
            c.advance(**kw)
    assert c.lens.tolist() == [10, 0, 90]
