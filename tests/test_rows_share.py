"""Rows that may share memory (rows.share), on the CPU."""
import pytest
import torch

from paper_2605_24259_amd.rows import moves, share


@pytest.mark.parametrize("rows,heads,dim", [(1, 1, 8), (3, 2, 8), (4, 1, 16)])
def test_sharing_is_found(rows, heads, dim):
    """Against the elements themselves; some layouts that share none may be refused, ordinary ones are not."""
    flat = torch.zeros(400)
    found = 0
    for row in (8, 16, 24, 32, 48):
        for head in (8, 16, 32):
            for other in (row, 40):
                for at in range(0, 200, 8):
                    a, b = flat.as_strided((rows, heads, dim), (row, head, 1), 96), flat.as_strided((rows, heads, dim), (other, head, 1), at)
                    flat.zero_()
                    a.fill_(1)
                    if b.any().item():
                        assert share(a, b) and share(b, a), (row, head, other, at)
                        found += 1
                    elif b.data_ptr() >= a[-1, -1].data_ptr() + 4 * dim and head * (heads - 1) < row * max(1, rows - 1):
                        assert not share(a, b), (row, head, other, at)
    assert found > 20 and not share(flat.view(1, 1, 400), torch.zeros(1, 1, 400))


def test_rows_in_their_own_place():
    x = torch.zeros(4, 6, 8)
    assert not moves(x, x) and not moves(x[:, :3], x[:, :3]) and not moves(x[:, :3], x[:, 3:]) and not moves(x[:2], x[2:])
    assert moves(x[:3], x[1:]) and moves(x[:, :3], x[:, 1:4]) and moves(x[:, :1], x.view(-1)[:32].view(4, 1, 8))
    # the stride of a dimension of one says nothing
    assert not moves(x[:1, :3], x.view(-1)[:24].view(1, 3, 8)) and not moves(x[1:2, 2:3], x[1, 2].view(1, 1, 8))
