"""Layer norm of the same rows in two layouts: what the kernel for aligned rows and the one for rows anywhere give, each against the plain form."""
import pytest
import torch

import paper_2505_11170_b200 as gws
from test_gpu_norm import check_backward, check_forward, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [96, 1365, 2048, 9000])
def test_copies_on_boundaries_and_rows_beside_them(n):
    m = 37
    room, weights = rand((m, n + 11), 1), rand((n + 1,), 4)
    x, r = room[:, 3:3 + n], rand((m * n + 1,), 3)[1:].view(m, n)
    dy, d = room.flip(0)[:, 1:1 + n], room[:, 7:7 + n]
    sides = []
    for copied in (False, True):
        a, b, c, e, w = (t.contiguous().clone() if copied else t for t in (x, r, dy, d, weights[1:]))
        y, s, stats = check_forward(a, w, None, b)
        sides.append((s, y, stats, *check_backward(c, s, w, stats, False, e)[:2]))
    assert torch.equal(sides[0][0], sides[1][0])               # the sum has one value; the others are within their bounds on either side
