"""CPU checks of the Python side of the training calls: what it refuses before any GPU work, how it
is built and what the package does without it."""
import pytest
import torch


def test_a_checkpoint_to_save_to_needs_a_save():
    """It used to be left as it was, in silence."""
    from paper_2108_08842_b200 import _binding

    native = _binding.native(0, 0, 0, 0, 0, 1)
    x, w = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(8, 32, dtype=torch.bfloat16)
    saved = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8)
    with pytest.raises(ValueError, match="saved is given"):
        _binding.linear(native, x, w, None, "none", None, None, "none", saved)


WITHOUT_BINDING = """
import sys
sys.path.insert(0, %r)
sys.modules["paper_2108_08842_b200._binding"] = None
from paper_2108_08842_b200 import eden
"""


def in_a_process(code):
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    return subprocess.run([sys.executable, "-c", WITHOUT_BINDING % root + code], capture_output=True, text=True, timeout=300)


def test_the_sender_is_there_without_the_extension():
    done = in_a_process("""
assert eden.code_bytes(1 << 20, 1.0) == 1 << 17 and eden.checkpoint_groups(33) == 2
ctx = object.__new__(eden.Context)
ctx._h, ctx._native = None, None
for call in (lambda: ctx.linear(1, 2), lambda: ctx.checkpoint_empty(1, 2), lambda: eden.eden_act_backward(ctx, 1, 2)):
    try:
        call()
    except ImportError as e:
        assert "_binding.so" in str(e)
    else:
        raise SystemExit("not refused")
""")
    assert done.returncode == 0, done.stderr


@pytest.mark.gpu
def test_rounds_without_the_extension():
    done = in_a_process("""
import torch
ctx = eden.Context(0, d_max=1 << 16, n_batch=2)
x = torch.randn((2, 1 << 16), device="cuda")
codes, scales = ctx.encode(x, [4.0, 4.0], [1, 2])
mean = ctx.mean(codes, scales, [4.0, 4.0], [1, 2], 1 << 16)
assert (mean - x.mean(dim=0)).norm() < 0.2 * x.mean(dim=0).norm() and ctx.status() == 0
ctx.close()
""")
    assert done.returncode == 0, done.stderr


# ------------------------------------------------------------------------------- the build
def test_the_command_builds_anew(monkeypatch, capsys):
    from paper_2108_08842_b200 import build

    calls = []
    monkeypatch.setattr(build, "build", lambda **how: calls.append(how) or "libeden.so")
    build.main()
    assert calls == [dict(force=True, verbose=True)] and capsys.readouterr().out == "libeden.so\n"


def test_a_failed_extension_is_named_and_the_library_is_there(monkeypatch, tmp_path):
    from paper_2108_08842_b200 import build

    build.build()                                        # the objects are there: only the link is left
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libeden.so"))
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_binding.so"))
    monkeypatch.setattr(build, "_binding_command", lambda out: ["false"])
    monkeypatch.setattr(build, "_fresh_binding", lambda: False)
    (tmp_path / "_binding.so").write_text("an older one")
    with pytest.raises(RuntimeError, match=r"g\+\+ failed building _binding.so"):
        build.build()
    assert (tmp_path / "libeden.so").exists() and not (tmp_path / "_binding.so").exists()


def test_an_extension_for_another_torch_is_stale(monkeypatch):
    from paper_2108_08842_b200 import _binding, build

    build.build()
    assert _binding.built_for == build.built_for() and torch.__version__ in build.built_for() and build._fresh_binding()
    monkeypatch.setattr(torch, "__version__", "1.0")
    assert not build._fresh_binding()


def test_an_extension_for_another_torch_is_not_used():
    done = in_a_process("""
import types
for name in [n for n in sys.modules if n.startswith("paper_2108_08842_b200")]:
    del sys.modules[name]
other = types.ModuleType("paper_2108_08842_b200._binding")
other.built_for = "torch 1.0, python 2.7"
sys.modules[other.__name__] = other
from paper_2108_08842_b200 import eden
try:
    eden._binding.linear
except ImportError as e:
    assert "torch 1.0" in str(e)
else:
    raise SystemExit("not refused")
""")
    assert done.returncode == 0, done.stderr
