"""What the operators' entry points refuse, through the C ABI and without a GPU. The context is a block of zeros: a call that gets past its
checks finds no device and returns SLIDEDP_ERR_CUDA."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would be made with an empty context")


@pytest.fixture(scope="module")
def sd():
    import paper_2609_34162_b200.slidedp as sd
    return sd


@pytest.fixture(scope="module")
def empty_context():
    return ctypes.create_string_buffer(1 << 14)


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


AT = 1 << 20          # an address that is aligned and never read


def norm_backward(sd, ctx, tokens, gate, gate_kind=1, dw_post=AT, dw_pre=AT, dgate=AT, workspace=AT):
    args = sd._BlockNormArgs(tokens=tokens, hidden=64, dtype=0, has_y=1, post_norm=1, pre_norm=1, gate_kind=gate_kind, gate_sigmoid=0,
                             residual_scale=1.0, eps=1e-6)
    rows = [ctypes.byref(Rows(AT * i, 64)) for i in range(1, 8)]
    x, y, dx_out, dh, dx, dy, none = rows
    return sd._lib.slidedp_block_norm_backward(ctx, ctypes.byref(args), x, y, None, gate, None, dx_out, dh, dx, dy,
                                               ctypes.byref(Rows(dgate, 64)) if dgate else None, dw_post, dw_pre, workspace, None)


@pytest.mark.parametrize("tokens", [0, 1])
def test_block_norm_backward_refuses_a_gate_that_is_not_there(sd, empty_context, tokens):
    accepted = ctypes.byref(Rows(9 * AT, 0))
    assert norm_backward(sd, empty_context, tokens, accepted) == sd.ERR_CUDA
    for gate in (None, ctypes.byref(Rows(None, 0)), ctypes.byref(Rows(9 * AT + 1, 0))):
        for wanted in (dict(), dict(dw_pre=None, dgate=None), dict(dw_post=None, dgate=None), dict(dw_post=None, dw_pre=None)):
            assert norm_backward(sd, empty_context, tokens, gate, **wanted) == sd.ERR_INVALID_ARG, (gate, wanted)
    assert norm_backward(sd, empty_context, tokens, None, gate_kind=0, dgate=None) == sd.ERR_CUDA
    assert norm_backward(sd, empty_context, tokens, accepted, workspace=None) == sd.ERR_INVALID_ARG
    assert norm_backward(sd, empty_context, tokens, accepted, workspace=AT + 4) == sd.ERR_MISALIGNED
