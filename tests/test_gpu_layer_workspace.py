"""Layer calls and their workspace: which calls need one, how large it may become, what is refused."""
import pytest
import torch

import paper_2009_09271_b200 as sc

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF16)


@pytest.mark.parametrize("rows", [1, 20, 70])
def test_column_sums_of_very_wide_rows(rows):
    """More strips of 256 columns than the tickets that joins of several runs of rows use."""
    cols = 4194304 + 257
    own = sc.Context(max_n=1)
    dy = normal(1, rows, cols)
    db = torch.empty(cols, device="cuda")
    own.sc_activation_grad(sc.SC_ACT_NONE, dy, None, None, None, db)
    want = dy.double().sum(0)
    assert bool(((db.double() - want).abs() <= (rows + 2) * 2.0 ** -23 * dy.double().abs().sum(0)).all())
    assert own.sc_sync_status() == 0
    own.close()
