"""Every pointer of the block operators' calls is refused where it is not
aligned to its element (no device is needed)."""
import ctypes

import pytest

import paper_1710_02368_amd as agn
from paper_1710_02368_amd import block
from tests.test_block_abi import GOOD, NORMS_GRAD, TYPES, P, _library

CASES = [("agn_dropout", ("x", "out", "step_dev")),
         ("agn_norms", ("residual", "f", "gate", "w_post", "w_pre", "step_dev", "residual_out", "h", "rstd_post",
                        "rstd_pre")),
         ("agn_route", ("logits", "chosen", "weights", "offsets", "source", "slot")),
         ("agn_route_backward", ("logits", "chosen", "weights", "dweights", "dlogits")),
         ("agn_dispatch", ("slot", "total", "x", "y")),
         ("agn_combine", ("slot", "total", "weights", "x", "y")),
         ("agn_combine_backward", ("slot", "total", "weights", "x", "y", "dy", "dweights")),
         ("agn_experts", ("offsets", "x", "w", "bias", "step_dev", "out")),
         ("agn_experts_backward", ("offsets", "x", "dy", "w", "dx", "dw", "dbias"))]


@pytest.mark.parametrize("name,field", [(n, f) for n, fields in CASES for f in fields])
def test_unaligned_pointers_are_refused(name, field):
    fields = dict(GOOD[name], **{field: P + 1})
    a = (TYPES.get(name) or getattr(block, name + "_args"))(**fields)
    assert getattr(_library(), name)(ctypes.addressof(a), None) == agn.AGN_EINVAL
    text = _library().agn_block_error().decode()
    assert "aligned" in text and (field in text or "not aligned to" in text), text


@pytest.mark.parametrize("field", ["dresidual_out", "dh", "dresidual", "df", "dgate", "dw_post", "dw_pre", "workspace",
                                   "rstd_post", "rstd_pre"])
def test_unaligned_pointers_of_the_norms_gradient_are_refused(field):
    fwd = dict(GOOD["agn_norms"], rstd_post=P, rstd_pre=P)
    grad = dict(NORMS_GRAD)
    (fwd if field.startswith("rstd") else grad)[field] = P + 1
    a = block.agn_norms_grad_args(block.agn_norms_args(**fwd), **grad)
    assert _library().agn_norms_backward(ctypes.addressof(a), None) == agn.AGN_EINVAL
    assert "aligned" in _library().agn_block_error().decode()
