"""The norms where a CTA goes through many rows: the last row numbers, further rounds of rows, and quantised rows of every kind."""
import pytest
import torch

import paper_2501_01144_b200 as bd

pytestmark = pytest.mark.gpu


def test_as_many_rows_as_there_can_be():
    rows, guard = 2 ** 31 - 1 - 128, 1 << 20
    y = torch.empty(rows + guard, dtype=torch.float16, device="cuda")
    for at in range(0, rows + guard, 1 << 28):
        part = y[at:at + (1 << 28)]
        part.copy_((torch.arange(at, at + part.numel(), device="cuda") % 1999).half())
    h = torch.full_like(y, 7.0)
    bd.residual_norm(y[guard:, None], None, scale=0.5, out_h=h[guard:, None])
    assert (h[:guard] == 7).all()
    for at in range(guard, rows + guard, 1 << 28):
        assert torch.equal(h[at:at + (1 << 28)], y[at:at + (1 << 28)] * 0.5)
    bd.poll_status()
