"""Rows that a write has no source for: the list names more rows than the call was given."""
import pytest
import torch

from test_gpu_cache import Pair, cu_of, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,cu", [(8, [0, 5, 9]), (6, [0, 7, 9]), (3, [0, 5, 9]), (4, [0, 5, 9]), (9, [-1, 5, 9])], ids=str)
def test_write_of_more_rows_than_given_is_reported(T, cu):
    """The rows that are there are written (those of [0, cu[n]) at their places), the missing ones are reported."""
    p = Pair(layers=1)
    p.reserve([0, 3], [6, 4]), p.check()
    x = torch.randn(2, T, 2, 64, generator=p.g).to(p.dt)
    y = x.to("cuda:0")
    p.c.write(y[0], y[1], ints([0, 3]), ints(cu), layer=0)
    for i, s in enumerate((0, 3)):
        for t in range(max(cu[i], 0), min(cu[i + 1], T)):
            at = int(p.b.len[s]) - (cu[i + 1] - t)
            if at < 0:                                                # more rows than the sequence has positions
                continue
            page, row = p.b.place(s, at)
            p.k[0, page, :, row], p.v[0, page, :, row] = x[0, t], x[1, t]
    p.check(7)


def test_write_of_exactly_the_rows_given_and_of_fewer():
    """Rows past the last list entry are not used, as in the attention calls."""
    p = Pair()
    p.reserve([0, 3], [5, 4])
    p.write([0, 3], [5, 4]), p.check()
    x = torch.ones(12, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    p.c.write(x, x, ints([0, 3]), cu_of([5, 4]), layer=0)
    for s, n in ((0, 5), (3, 4)):
        for j in range(n):
            page, row = p.b.place(s, j)
            p.k[0, page, :, row], p.v[0, page, :, row] = 1, 1
    p.check()
