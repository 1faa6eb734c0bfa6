"""What the norm, dropout and 8-bit operators refuse before any device is touched, and the statements that their GPU tests rest on."""
import pytest
import torch

import paper_2009_09271_b200 as sc
from block_util import SALT_DROPOUT, kept_mask, norm64, norm_grad64, rows_in_8_bits
from oracle import sparsify_oracle as O
from paper_2009_09271_b200 import binding


def test_quantized_buffers():
    q, s = sc.quantized_buffers(3, 40, device="cpu")
    assert q.shape == (3, 40) and q.dtype == torch.int8 and s.shape == (3,) and s.dtype == torch.float32


def test_eight_bit_rows_are_both_tensors():
    q, s = sc.quantized_buffers(3, 40, device="cpu")
    for bad in ((q, None), (None, s)):
        with pytest.raises(ValueError):
            binding._eight_bit_rows(*bad, 3, 40)
    with pytest.raises(TypeError):
        binding._eight_bit_rows(q, s, 3, 40)                            # on the host


def test_probabilities():
    for p in (0, 0.0, 0.5, 1, 1.0):
        assert binding._probability(p) == p
    for p in (-1e-9, 1.0000001, float("nan"), float("inf")):
        with pytest.raises(ValueError):
            binding._probability(p)


CALLS = (("sc_quantize", (None, 0, None, 0, 0, 0, None, 0, None, None)),
         ("sc_dequantize", (None, 0, None, 0, None, 0, 0, None, 0, None)),
         ("sc_linear_quantized", (None, 0, 0, None, 0, None, None, 0, None, None, None, 0, 0, 0, 0, None, 0, None, None, None)),
         ("sc_dropout", (None, 0, None, 0, None, 0, 0.5, 2 ** 64 - 1, 0, 0, None, 0, None)),
         ("sc_rms_norm", (None, 0, None, 0, None, 0, None, 1e-6, 0.5, 3, 0, 0, None, 0, None, 0, None, 0, None, None)),
         ("sc_rms_norm_grad", (None, 0, None, 0, None, 0, None, 1e-6, None, 0, 0.5, 3, 0, 0, None, 0, None, 0, None, 0, None)))


@pytest.mark.parametrize("name,args", CALLS)
def test_null_context_and_wrong_arguments(name, args):
    lib = sc.load_library()
    calls = binding._layer_calls(lib)
    assert getattr(lib, name)(*args) == getattr(calls, name)(*args) == -1
    if calls is not lib:
        for bad in (args[:-1], args + (None,), args[:1] + ("0",) + args[2:]):
            with pytest.raises((TypeError, OverflowError)):
                getattr(calls, name)(*bad)


def test_tensors_are_taken_by_a_caller_built_for_this_torch_only():
    import types
    here = torch.__version__.split("+")[0]
    calls = binding._layer_calls(sc.load_library())
    if hasattr(calls, "bind"):
        assert calls.torch_version.split("+")[0] == here and binding._tensor_calls(calls) is calls
    for built_for, taken in ((here, True), (here + "+cu1", True), ("1.0.0", False), (here + "1", False)):
        fake = types.SimpleNamespace(torch_version=built_for)
        assert binding._tensor_calls(fake) is (fake if taken else None)
    assert binding._tensor_calls(types.SimpleNamespace()) is None and binding._tensor_calls(object()) is None


def test_kept_mask_is_the_oracles_generator():
    for seed, rows, cols, p in ((0, 3, 7, 0.5), (2 ** 64 - 5, 2, 8, 0.1), (12345, 1, 1, 0.9)):
        mask, scale = kept_mask(seed, rows, cols, p)
        key, cut = O.mix64(seed, SALT_DROPOUT), round(p * 65536)
        for i in range(rows):
            for j in range(cols):
                word = O.mix64(key, i * -(-cols // 4) + j // 4)
                assert bool(mask[i, j]) == ((word >> (16 * (j % 4)) & 0xFFFF) >= cut)
        assert scale == 65536 / (65536 - cut)


def test_rows_in_8_bits_by_hand():
    q, s = rows_in_8_bits(torch.tensor([[127.0, -63.5, 0.5, 1.5], [0.0, 0.0, 0.0, 0.0], [1.0, float("nan"), 0.0, 0.0], [2.0 ** -101, 0.0, 0.0, 0.0]]))
    assert q.tolist() == [[127, -64, 0, 2], [0] * 4, [0] * 4, [0] * 4]
    assert s[0] == 1 and s[1] == 0 and bool(torch.isnan(s[2])) and s[3] == 0


def test_norm_statements_agree_with_automatic_differentiation():
    g = torch.Generator().manual_seed(1)
    x, c, gamma = (torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True) for s in ((5, 12), (5, 12), (12,)))
    h, y = norm64(x, None, gamma, 1e-3)
    y.backward(c.detach())
    (dh, dgamma), _ = norm_grad64(c.detach(), x.detach(), gamma.detach(), 1e-3)
    assert torch.allclose(dh, x.grad, atol=1e-12) and torch.allclose(dgamma, gamma.grad, atol=1e-12)
