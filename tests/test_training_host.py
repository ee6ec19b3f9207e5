"""CPU checks of the training entry points: size rules, argument checks before any GPU work."""
import ctypes
import struct

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
        assert b > last and b >= 2 * 2 * size * size
        last = b


NAMES = ("eden_linear", "eden_checkpoint_save", "eden_checkpoint_restore", "eden_act_backward", "eden_linear_input_grad",
         "eden_linear_weight_grad")


@pytest.mark.parametrize("name", NAMES)
def test_null_arguments_are_refused(lib, name):
    fn = getattr(lib, name)
    fn.argtypes = [ctypes.c_void_p, ctypes.c_char_p]
    assert fn(None, b"\0" * 256) == -1
    assert fn(None, None) == -1


def test_binding_lays_out_the_argument_blocks_as_the_header_does():
    import os
    import subprocess
    import tempfile

    from paper_2108_08842_b200 import eden

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {"eden_linear_args": ("m", "reserved", eden._LINEAR, 13), "eden_checkpoint_args": ("m", "reserved", eden._CHECKPOINT, 6),
              "eden_act_backward_args": ("m", "reserved", eden._ACT_BACKWARD, 9),
              "eden_linear_input_grad_args": ("m", "reserved", eden._INPUT_GRAD, 13),
              "eden_linear_weight_grad_args": ("m", "accumulate", eden._WEIGHT_GRAD, 10)}
    body = "".join('printf("%%zu %%zu %%zu\\n", sizeof(%s), offsetof(%s, %s), offsetof(%s, %s));' % (s, s, f[0], s, f[1]) for s, f in fields.items())
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "a.c"), os.path.join(d, "a")
        with open(src, "w") as f:
            f.write('#include "%s"\n#include <stddef.h>\n#include <stdio.h>\nint main(void){%s return 0;}' % (os.path.join(root, "include", "eden.h"), body))
        subprocess.run(["gcc", "-o", exe, src], check=True)
        rows = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    rows = [tuple(map(int, rows[i:i + 3])) for i in range(0, len(rows), 3)]
    for (_, _, block, count_at), (size, at, last) in zip(fields.values(), rows):
        assert block.size == size and struct.calcsize("@%dQ" % count_at) == at and last == size - 4
