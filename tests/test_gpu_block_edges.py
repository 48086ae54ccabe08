"""The block operators at the edges of their arguments' ranges, and on every
kernel that their rules choose between."""
import numpy as np
import pytest
import torch

from tests import block_oracle as O
from tests.block_kernels import CASES
from tests.helpers import require_gpu
from tests.test_gpu_block import BOTH, DTYPES, SEED, _check_experts, _check_norms, _norms_case

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


# ---------------------------------------------------------------------------
# infinities under the mask
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("what", ["gate", "w_post"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@BOTH
@pytest.mark.parametrize("cols", [64, 517, 5000])
def test_norms_factors_of_dropped_elements(cols, dtype, value, what):
    """A dropped element is 0 whatever its factors are: an infinite or NaN gate
    or weight there gives the bits of a finite one, in both directions.  (w_post
    is a value a column: one row, so that no kept element has it.)"""
    block = _block()
    rows, rate = (6, 0.4) if what == "gate" else (1, 0.4)
    keep = O.mask(rows, cols, rate, SEED, 3)
    g = torch.Generator().manual_seed(cols)
    rand = lambda *s: torch.randn(*s, generator=g)
    r, f, dres, dh, gate = (rand(rows, cols).to(DTYPES[dtype]).cuda() for _ in range(5))
    w_post, w_pre = (1 + 0.1 * rand(cols)).cuda(), (1 + 0.1 * rand(cols)).cuda()
    dropped = (keep == 0).cuda()
    assert dropped.any() and not dropped.all()

    def both(gate, w_post):
        kw = dict(gate=gate, alpha=0.5, dropout=(rate, SEED, 3))
        res, h, saved = block.norms(r, f, w_post, w_pre, **kw)
        return (res, h, *block.norms_backward(dres, dh, res, f, w_post, w_pre, saved, **kw))

    want = both(gate, w_post)
    if what == "gate":
        got = both(torch.where(dropped, value, gate.float()).to(DTYPES[dtype]), w_post)
    else:
        got = both(gate, torch.where(dropped[0], value, w_post))
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.isfinite(b).all() and torch.equal(a, b), i


@BOTH
@pytest.mark.parametrize("rows,cols", [(1100, 4096), (1100, 4100), (700, 8192), (1300, 2056)])
@pytest.mark.parametrize("gate", ["channel", "full"])
def test_norms_many_wide_rows(rows, cols, gate, dtype):
    """Teams of 8 and 16 waves that walk several rows each."""
    _check_norms(_block(), *_norms_case(rows, cols, dtype, gate), 0.1, dtype)


# ---------------------------------------------------------------------------
# the experts' products: more experts than a wave has lanes
# ---------------------------------------------------------------------------

def _mostly_the_last(experts, rows):
    """Two rows to the first expert, one to the 64th, the rest to the last two."""
    counts = [0] * experts
    counts[0], counts[63], counts[-2] = 2, 1, (rows - 3) // 3
    counts[-1] = rows - sum(counts)
    return counts


@BOTH
@pytest.mark.parametrize("experts", [65, 130, 1024])
@pytest.mark.parametrize("rows,i,o", [(64, 200, 72), (300, 72, 130), (800, 40, 72)])
def test_many_experts(experts, rows, i, o, dtype):
    """Few rows and many, nearly all of them in the last group of 64 experts."""
    counts = _mostly_the_last(experts, rows - 5)
    _check_experts(_block(), rows, counts, i, o, True, 0.1, "plain", dtype)


@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}_{c[1]}rows_{len(c[2])}e_{c[3]}x{c[4]}" for c in CASES])
def test_every_kernel_of_the_experts(case):
    dtype, rows, counts, i, o = case
    rate = 0.1 if rows * o < 1 << 21 else 0.0
    _check_experts(_block(), rows, counts, i, o, True, rate, "plain", dtype)


@BOTH
def test_experts_of_many_rows_do_not_mix_rows(dtype):
    """As with few rows: NaN and infinities of one expert's rows stay in its
    outputs, in the tiles' kernels, aligned, odd and shorter than a load."""
    block = _block()
    for i, o in ((72, 40), (75, 41), (256, 256), (5, 300), (3, 300)):
        counts = [330, 235, 220]
        x, w, dy = (torch.randn(*s, generator=torch.Generator().manual_seed(n)).to(DTYPES[dtype]).cuda()
                    for n, s in enumerate(((800, i), (3, o, i), (800, o))))
        x[330:565], x[785:], dy[330:565], dy[785:] = float("nan"), float("inf"), float("inf"), float("nan")
        off = torch.tensor([0, *np.cumsum(counts)], dtype=torch.int32, device="cuda")
        h = block.experts(x, off, w)
        dx, dw, db = block.experts_backward(x, dy, off, w)
        for v in (h, dx):
            assert torch.isfinite(v[:330]).all() and torch.isfinite(v[565:785]).all() and (v[785:] == 0).all()
            assert not torch.isfinite(v[330:565]).any()
        for v in (dw, db):
            assert torch.isfinite(v[[0, 2]]).all() and not torch.isfinite(v[1]).any()


# ---------------------------------------------------------------------------
# beside autograd
# ---------------------------------------------------------------------------

def test_writing_in_place_counts_as_a_modification():
    """A tensor that autograd saved and dropout then wrote over must not be used
    in the backward pass; one that requires gradients is not written over."""
    block = _block()
    w = torch.ones(8, 8, device="cuda", requires_grad=True)
    x = torch.ones(8, 8, device="cuda")
    y = (w * x).sum()
    block.dropout(x, 0.5, SEED, 0, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    out = torch.empty(8, 8, device="cuda")
    before = out._version
    block.dropout(w, 0.5, SEED, 0, out=out)
    assert out._version == before + 1 and not out.requires_grad
    with pytest.raises(ValueError, match="out requires gradients"):
        block.dropout(x, 0.5, SEED, 0, out=w)
    assert (w == 1).all()
    with torch.no_grad():
        block.dropout(x, 0.5, SEED, 0, out=w)
    assert torch.equal(w.detach(), block.dropout(x, 0.5, SEED, 0))
