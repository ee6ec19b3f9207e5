"""CPU checks of joins and 4-bit products: size rules, and what is refused before any GPU work."""
import ctypes

import pytest
import torch

NAMES = ("eden_block_join", "eden_block_join_backward", "eden_mx4_quantize", "eden_mx4_restore", "eden_mx4_linear", "eden_mx4_linear_input_grad",
         "eden_mx4_linear_weight_grad")


@pytest.fixture(scope="module")
def lib():
    from paper_2108_08842_b200 import build

    return ctypes.CDLL(build.build())


@pytest.mark.parametrize("name", NAMES)
def test_null_arguments_are_refused(lib, name):
    fn = getattr(lib, name)
    fn.argtypes = [ctypes.c_void_p, ctypes.c_char_p]
    assert fn(None, b"\0" * 512) == -1
    assert fn(None, None) == -1


def test_size_rules(lib):
    from paper_2108_08842_b200 import eden

    for name, count in (("eden_mx4_code_bytes", 1), ("eden_mx4_exponent_bytes", 2)):
        getattr(lib, name).restype, getattr(lib, name).argtypes = ctypes.c_uint64, [ctypes.c_uint64] * count
    assert [lib.eden_mx4_code_bytes(n) for n in (1, 32, 33, 4096)] == [16, 16, 32, 2048]
    assert [lib.eden_mx4_exponent_bytes(*s) for s in ((1, 1), (128, 256), (129, 256), (128, 257), (0, 5))] == [1024, 1024, 2048, 2048, 0]
    last = 0
    for size in (1, 100, 1000, 5000, 70000):
        need = eden.mx4_workspace_bytes(size, size, size)
        assert need >= last and need >= size * size // 2
        last = need
        assert eden.block_workspace_bytes(size) >= 4 * 512 * size


@pytest.fixture(scope="module")
def native():
    from paper_2108_08842_b200 import _binding

    return _binding.native(0, 0, 0, 0, 0, 1)


def test_joins_refuse(native):
    """On CPU tensors: the checks come before the library is called."""
    from paper_2108_08842_b200 import _binding, eden

    h = torch.zeros(4, 32, dtype=torch.bfloat16)
    tail = (None, 1.0, 0.0, 0, 0, None, None, False)
    for bad in (lambda: _binding.join(native, h, None, None, None, *tail), lambda: _binding.join(native, None, None, None, None, *tail),
                lambda: _binding.join(native, h.float(), None, None, None, *tail), lambda: _binding.join(native, h[0], None, None, None, *tail),
                lambda: _binding.join_backward(native, None, None, h, h, *[None] * 5, 1.0, 0.0, 0, 0, *[None] * 7, False),
                lambda: _binding.join_backward(native, h, None, h, h, *[None] * 5, 1.0, 0.0, 0, 0, *[None] * 7, False)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        _binding.join(native, h)
    assert eden.Norm().kind == "rms" and eden.Norm(kind="layer").weight is None


def test_4_bit_calls_refuse(native):
    from paper_2108_08842_b200 import _binding, eden

    x, codes, exps = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(1, 1, 1024, dtype=torch.uint8)
    q = eden.Mx4(codes, exps, 32)
    for bad in (lambda: _binding.mx4_empty(native, -1, 4), lambda: _binding.mx4_empty(native, 4, 0), lambda: _binding.mx4_quantize(native, x, None, False),
                lambda: _binding.mx4_quantize(native, x.double(), None, False), lambda: _binding.mx4_restore(native, q, torch.int8, None),
                lambda: _binding.mx4_restore(native, q, torch.float32, None), lambda: _binding.mx4_restore(native, x, torch.float32, None),
                lambda: _binding.mx4_restore(native, (codes, exps), torch.float32, None), lambda: _binding.mx4_restore(native, eden.Mx4(codes, exps, 0), torch.float32, None),
                lambda: _binding.mx4_restore(native, eden.Mx4(codes, exps, "32"), torch.float32, None),
                lambda: _binding.mx4_linear(native, x, x, None, "none", None, None, "none", None, None),
                lambda: _binding.mx4_linear(native, x, q, None, "none", None, None, "none", None, None),
                lambda: _binding.mx4_input_grad(native, x, q, None, None, "none", None, None, False, None),
                lambda: _binding.mx4_weight_grad(native, q, q, None, False), lambda: _binding.mx4_weight_grad(native, x, x, None, False)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.gpu
def test_calls_of_a_context_refuse():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.mx4_workspace_bytes(64, 64, 64) + eden.block_workspace_bytes(64))
    dev = dict(dtype=torch.bfloat16, device="cuda")
    h, v, s = torch.zeros(8, 64, **dev), torch.ones(64, **dev), torch.zeros(8, 2, device="cuda")
    norm = eden.Norm(v)
    wide = torch.zeros(2, eden_max() + 1, **dev)
    join, back = c.block_join, c.block_join_backward
    for bad in (lambda: join(h, h.half()), lambda: join(h, h[:4]), lambda: join(h.t()), lambda: join(h, after=v), lambda: join(h, after=eden.Norm(v[:32])),
                lambda: join(h, after=eden.Norm(v.half())), lambda: join(h, after=eden.Norm(v.cpu())), lambda: join(h, after=eden.Norm(v, kind="batch")),
                lambda: join(h, after=eden.Norm(v, eps=-1.0)), lambda: join(h, after=eden.Norm(v, eps=float("nan"))), lambda: join(h, after=eden.Norm(v, eps="1")),
                lambda: join(h, gate=v[:8]), lambda: join(h, gate=h[:4]), lambda: join(h, drop=-0.1), lambda: join(h, drop=1.5), lambda: join(h, drop=float("nan")),
                lambda: join(h, drop=0.5, seed=-1), lambda: join(h, drop=0.5, seed=2 ** 64), lambda: join(h, drop=0.5, seed=1.5),
                lambda: join(h, drop=0.5, seed=torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: join(h, drop=0.5, seed=torch.zeros(1, dtype=torch.int64)),
                lambda: join(h, drop=0.5, seed=torch.zeros(1, dtype=torch.int32, device="cuda")), lambda: join(h, drop=0.5, first_row=-1), lambda: join(h, out=False),
                lambda: join(h, out=h[:4]), lambda: join(h, normed=h), lambda: join(h, before=norm, normed=h.float()), lambda: join(h, before=norm, normed=False),
                lambda: back(None, None), lambda: back(h, h), lambda: back(h, None, before=norm), lambda: back(h, h, before=norm), lambda: back(h, h, x=h, before=norm),
                lambda: back(h, h, x=h, before=norm, before_stats=s[:4]), lambda: back(h, h, x=h, before=norm, before_stats=s.half()), lambda: back(h, None, after=norm),
                lambda: back(h, None, h, after=norm), lambda: back(h, None, gate=v), lambda: back(h, None, h=h.float(), gate=v), lambda: back(h, None, h=(h, h), gate=v),
                lambda: back(h, None, gate_grad=v.float()), lambda: back(h, None, h=h, gate=v, gate_grad=v), lambda: back(h, None, after_weight_grad=v.float()),
                lambda: back(h, None, h=h, after=norm, after_stats=s, accumulate=True), lambda: c.norm(h, None), lambda: c.dropout(h, 2.0, 1)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: c.norm(wide, eden.Norm()), lambda: join(h, scale=float("inf")), lambda: join(h, drop=0.5, first_row=2 ** 32 - 4)):
        with pytest.raises(eden.EdenError):
            bad()
    assert torch.equal(c.dropout(wide, 0.0, 1), wide)                    # without norms rows may be longer

    q, w = c.mx4_quantize(h), c.mx4_quantize(torch.zeros(32, 64, **dev))
    bytes_ = torch.zeros(8 * 33, dtype=torch.uint8, device="cuda")
    shifted = eden.Mx4(bytes_[1:257].view(8, 32), q.exps, 64)
    pitch = eden.Mx4(bytes_.view(8, 33)[:, :32], q.exps, 64)
    for bad in (lambda: c.mx4_linear(h, h), lambda: c.mx4_linear(h[:, :32], w), lambda: c.mx4_linear(h.float(), w), lambda: c.mx4_linear(q, w, dtype=torch.float32),
                lambda: c.mx4_linear(h, w, dtype=torch.float16), lambda: c.mx4_linear(shifted, w), lambda: c.mx4_linear(pitch, w), lambda: c.mx4_linear(q._replace(features=63), w),
                lambda: c.mx4_linear(q._replace(features=65), w), lambda: c.mx4_linear(q._replace(exps=q.exps[:, :, :512]), w),
                lambda: c.mx4_linear(q._replace(codes=q.codes.to(torch.int8)), w), lambda: c.mx4_linear(q._replace(codes=q.codes.cpu()), w),
                lambda: c.mx4_linear(q, w, v), lambda: c.mx4_linear(q, w, act="tanh"), lambda: c.mx4_linear(q, w, save="none", saved=c.checkpoint_empty(8, 32)),
                lambda: c.mx4_linear(q, w, out=h), lambda: c.mx4_quantize(h, w), lambda: c.mx4_quantize_transposed(h, q), lambda: c.mx4_quantize_transposed(h[:0]),
                lambda: c.mx4_restore(q, torch.bfloat16, h.half()), lambda: c.mx4_linear_input_grad(q, w, act="gelu"), lambda: c.mx4_linear_input_grad(q, w, accumulate=True),
                lambda: c.mx4_linear_input_grad(q, w, pre=c.checkpoint_empty(8, 64)), lambda: c.mx4_linear_weight_grad(q, w, accumulate=True),
                lambda: c.mx4_linear_weight_grad(q, q._replace(features=32)), lambda: c.mx4_linear_weight_grad(q, w, out=h)):
        with pytest.raises(ValueError):
            bad()
    assert c.status() == 0
    c.close()


def eden_max():
    return 32768


def test_options_of_the_client_are_checked():
    from paper_2108_08842_b200 import client

    for bad in (dict(norm="batch"), dict(products="int4"), dict(drop=0.1), dict(gate=True), dict(products="mx4")):
        with pytest.raises(ValueError):
            client.FeedForward(None, 32, 64, **bad)
