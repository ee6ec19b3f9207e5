"""CPU checks of the training entry points: size rules, argument checks before any GPU work."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2108_08842_b200 import build
    handle = ctypes.CDLL(build.build())
    handle.eden_checkpoint_groups.restype = ctypes.c_uint64
    handle.eden_checkpoint_groups.argtypes = [ctypes.c_uint64]
    handle.eden_linear_workspace_bytes.restype = ctypes.c_uint64
    handle.eden_linear_workspace_bytes.argtypes = [ctypes.c_uint64] * 3
    return handle


def test_size_rules(lib):
    assert [lib.eden_checkpoint_groups(n) for n in (0, 1, 31, 32, 33, 4096)] == [0, 1, 1, 1, 2, 128]
    last = 0
    for size in (1, 8, 100, 1000, 5000):
        b = lib.eden_linear_workspace_bytes(size, size, size)
        assert b >= last and b >= 2 * 2 * size * size
        last = b


NAMES = ("eden_linear", "eden_checkpoint_save", "eden_checkpoint_restore", "eden_act_backward", "eden_linear_input_grad",
         "eden_linear_weight_grad")


@pytest.mark.parametrize("name", NAMES)
def test_null_arguments_are_refused(lib, name):
    fn = getattr(lib, name)
    fn.argtypes = [ctypes.c_void_p, ctypes.c_char_p]
    assert fn(None, b"\0" * 256) == -1
    assert fn(None, None) == -1


def test_calls_of_a_context_refuse_before_any_gpu_work():
    """Argument checks of the binding on CPU tensors: they come before the library is called."""
    import torch

    from paper_2108_08842_b200 import _binding

    native = _binding.native(0, 0, 0, 0, 0, 1)
    x, w = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(8, 32, dtype=torch.bfloat16)
    for bad in (lambda: _binding.linear(native, x, w, None, "none", None, None, "none", None),
                lambda: _binding.linear(native, x, None, None, "none", None, None, "none", None),
                lambda: _binding.linear(native, x[0], w, None, "none", None, None, "none", None),
                lambda: _binding.linear(native, x.float(), w, None, "none", None, None, "none", None),
                lambda: _binding.linear(native, x, w, None, "tanh", None, None, "none", None),
                lambda: _binding.linear(native, x, w, None, None, None, None, "none", None),
                lambda: _binding.linear(native, x, w, None, "none", None, None, 3, None),
                lambda: _binding.checkpoint_empty(native, -1, 4),
                lambda: _binding.checkpoint_save(native, x.double(), None),
                lambda: _binding.checkpoint_restore(native, (x, x), torch.int8, None),
                lambda: _binding.checkpoint_restore(native, [x, x], torch.float32, None),
                lambda: _binding.act_backward(native, x, None, "gelu", None, None, False),
                lambda: _binding.input_grad(native, x, w, None, None, "relu", None, None, False),
                lambda: _binding.weight_grad(native, x, (x,), None, False)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        _binding.linear(native, x, w)
    with pytest.raises(ValueError):
        _binding.linear("native", x, w, None, "none", None, None, "none", None)
