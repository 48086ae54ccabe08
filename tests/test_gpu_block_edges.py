"""The block operators at the edges of their arguments' ranges, and on every
kernel that their rules choose between."""
import numpy as np
import pytest
import torch

from tests import block_oracle as O
from tests.helpers import require_gpu
from tests.test_gpu_block import SEED

pytestmark = pytest.mark.gpu


def _block():
    require_gpu()
    from paper_1710_02368_amd import block
    return block


# ---------------------------------------------------------------------------
# the widest rows
# ---------------------------------------------------------------------------

WIDEST = [(1 << 31) - 1, (1 << 31) - 8, (1 << 31) - 2040]


def _wide_row(cols):
    """One bfloat16 row of small whole numbers that are not zero."""
    i = torch.arange(cols, dtype=torch.int32, device="cuda")
    return ((i & 127) + 1).to(torch.bfloat16).reshape(1, cols)


def _keep(c, rate, step):
    """The scaled mask of row 0 at columns c."""
    t = O.threshold(rate)
    c = np.asarray(c, dtype=np.uint64)
    w = O.philox((c >> np.uint64(3), 0, 0, step), (SEED & 0xFFFFFFFF, SEED >> 32))
    w = np.stack([np.broadcast_to(v, c.shape) for v in w])
    word = w[(c & np.uint64(7)) >> np.uint64(1), np.arange(c.size)]
    draw = np.where(c & np.uint64(1), word >> np.uint64(16), word & np.uint64(0xFFFF))
    return (draw >= t) * (65536.0 / (65536 - t))


@pytest.mark.parametrize("cols", WIDEST)
def test_dropout_of_the_widest_rows(cols):
    """Rows of up to 2^31 - 1 columns, the counter's and the chunks' last ones among them."""
    block = _block()
    x = _wide_row(cols)
    y = block.dropout(x, 0.5, SEED, 2)
    at = np.concatenate([np.arange(2000), np.arange(cols // 2 - 1000, cols // 2 + 1000), np.arange(cols - 3000, cols)])
    pick = torch.from_numpy(at).cuda()
    want = x[0, pick].double().cpu().numpy() * _keep(at, 0.5, 2)
    np.testing.assert_array_equal(y[0, pick].double().cpu().numpy(), want)  # (a product by 2: exact)
    kept = (y != 0).sum().item()
    assert abs(kept / cols - 0.5) < 6 * 0.5 / cols ** 0.5


@pytest.mark.parametrize("cols", WIDEST)
def test_tokens_of_the_widest_rows(cols):
    """One row to the second of its two choices (the first is no expert), and
    back; the other place is cleared to its last column."""
    block = _block()
    x = _wide_row(cols)
    r = block.route_chosen(torch.tensor([[-1, 2]], dtype=torch.int32, device="cuda"),
                           torch.tensor([[9.0, 0.5]], device="cuda"), 3)
    y = block.dispatch(x, r)
    assert torch.equal(y[0], x[0]) and not y[1].any()
    back = block.combine(y, r)
    assert torch.equal(back, x * 0.5)
