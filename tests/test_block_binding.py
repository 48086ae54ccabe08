"""What the block operators' binding refuses before it reaches the library
(no device is needed: the arguments are looked at first)."""
import pytest
import torch

from paper_1710_02368_amd import block


def _meta(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("cols", [1 << 31, 1 << 32, (1 << 32) + 8])
def test_widths_that_the_structs_cannot_hold(cols):
    """A width of 2^32 + 8 would arrive as 8, and most of the output would stay unwritten."""
    for call in (lambda: block.dropout(_meta(1, cols), 0.1, 1, 1),
                 lambda: block.norms(_meta(1, cols), None, None, None),
                 lambda: block.route(_meta(1, cols), 2),
                 lambda: block.dispatch(_meta(1, cols), None),
                 lambda: block.experts(_meta(1, cols), None, None)):
        with pytest.raises(ValueError, match="fewer than 2\\^31 columns"):
            call()
    for shape in ((1, 1, cols), (1, cols, 1), (cols, 1, 1)):
        with pytest.raises(ValueError, match="w: every size"):
            block._experts_weights(_meta(*shape), _meta(1, 1))


class Device(torch.Tensor):
    """Stands for a tensor on the device."""
    is_cuda = True


@pytest.mark.parametrize("n", [-1, 1 << 31, (1 << 32) + 2])
def test_counts_that_the_structs_cannot_hold(n):
    with pytest.raises(ValueError, match="k must be in"):
        block.route(_meta(4, 8).as_subclass(Device), n)
    with pytest.raises(ValueError, match="experts must be in"):
        block.route_chosen(_meta(4, 2, dtype=torch.int32).as_subclass(Device), None, n)


@pytest.mark.parametrize("offsets", [torch.empty(0, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                                     torch.zeros(2, 2, dtype=torch.int32)], ids=["empty", "one", "matrix"])
def test_offsets_without_a_last_one(offsets):
    """The count of places in use is read from the last of experts + 1 offsets."""
    slot = torch.zeros(3, 2, dtype=torch.int32)
    r = block.Route(slot, None, offsets, slot.reshape(-1), slot)
    x = torch.zeros(3, 8)
    with pytest.raises(ValueError, match="offsets"):
        block._tokens("agn_dispatch", r, 3, 8, (x.data_ptr(), 8), (x.data_ptr(), 8), x, False)


def test_gradients_of_what_is_not_there():
    """Choices without weights, norms before a block without the gradient of their output."""
    chosen = _meta(3, 2, dtype=torch.int32)
    logits = _meta(3, 8, dtype=torch.float32).as_subclass(Device)
    r = block.Route(chosen, None, _meta(9, dtype=torch.int32), chosen.reshape(-1), chosen)
    with pytest.raises(ValueError, match="no weights"):
        block.route_backward(logits, r, _meta(3, 2, dtype=torch.float32))
    x, w = _meta(3, 8, dtype=torch.float32).as_subclass(Device), _meta(8, dtype=torch.float32)
    saved = block.NormsSaved(_meta(2, 3, dtype=torch.float32), x)
    with pytest.raises(ValueError, match="dh must"):
        block.norms_backward(None, None, x, None, None, w, saved)


def test_every_public_name_is_listed():
    own = {n for n, v in vars(block).items() if not n.startswith(("_", "agn_")) and callable(v)
           and getattr(v, "__module__", "") == block.__name__}
    assert own == set(block.__all__) - {"EXPORTED"}
