"""What the layer operators' binding refuses before any device is touched."""
import pytest
import torch

import paper_2009_09271_b200 as sc
from paper_2009_09271_b200 import binding


def test_checkpoint_buffers_cover_ragged_groups():
    for rows, cols in ((1, 1), (3, 32), (5, 33), (0, 64), (7, 1000)):
        q, scales = sc.checkpoint_buffers(rows, cols, device="cpu")
        assert q.shape == (rows, cols) and q.dtype == torch.int8
        assert scales.shape == (rows, -(-cols // sc.CHECKPOINT_GROUP)) and scales.dtype == torch.uint8


def test_activation_names():
    assert sc.ACTIVATIONS == {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


@pytest.mark.parametrize("bad", [torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(32, dtype=torch.bfloat16)])
def test_matrix_refuses_host_tensors_other_types_and_shapes(bad):
    with pytest.raises(TypeError):
        binding._matrix(bad, 4, 8, torch.bfloat16, "x")


def test_layer_type_refuses_what_the_products_do_not_take():
    assert binding._layer_type(torch.zeros(2, 2, dtype=torch.float16), "x") == sc.SC_F16
    assert binding._layer_type(torch.zeros(2, 2), "x", f32=True) == sc.SC_F32
    with pytest.raises(TypeError):
        binding._layer_type(torch.zeros(2, 2), "x")
    with pytest.raises(TypeError):
        binding._layer_type(torch.zeros(2, 2, dtype=torch.float64), "x", f32=True)
    with pytest.raises(ValueError):
        binding._layer_type(torch.zeros(2, dtype=torch.bfloat16), "x")


def test_a_checkpoint_is_both_tensors():
    q, scales = sc.checkpoint_buffers(2, 40, device="cpu")
    with pytest.raises(ValueError):
        binding._kept(q, None, 2, 40)
    with pytest.raises(ValueError):
        binding._kept(None, scales, 2, 40)


def test_null_context_is_an_error_code():
    lib = sc.load_library()
    assert lib.sc_layer_reserve(None, 1, 1, 1) == -1
    assert lib.sc_checkpoint_pack(None, 0, None, 0, 0, 0, None, None, None) == -1
    assert lib.sc_linear_grad_weight(None, 0, None, 0, None, 0, None, None, 0, 0, 0, None, 0, 0, None) == -1


def test_compiled_calls_agree_with_ctypes():
    """The compiled caller and ctypes reach the same functions with the same arguments: argument errors come back alike."""
    lib = sc.load_library()
    calls = binding._layer_calls(lib)
    for name, args in (("sc_checkpoint_pack", (None, 0, None, 0, 0, 0, None, None, None)),
                       ("sc_checkpoint_unpack", (None, 0, None, None, 0, 0, None, 0, None)),
                       ("sc_activation_grad", (None, 0, 0, None, 0, None, None, 0, 0, None, 0, None, 0, None)),
                       ("sc_linear", (None, 0, 0, None, 0, None, 0, None, None, 0, 0, 0, 0, None, 0, None, None, None)),
                       ("sc_linear_grad_input", (None, 0, 0, None, 0, None, 0, None, 0, None, None, 0, 0, 0, None, 0, None)),
                       ("sc_linear_grad_weight", (None, 0, None, 0, None, 0, None, None, 0, 0, 0, None, 0, 0, None))):
        assert getattr(calls, name)(*args) == getattr(lib, name)(*args) == -1
        if calls is not lib:
            with pytest.raises(TypeError):
                getattr(calls, name)(*args[:-1])
            with pytest.raises((TypeError, OverflowError)):
                getattr(calls, name)(*args[:1], "0", *args[2:])
