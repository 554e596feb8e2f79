"""The extension behind the operators on whole sets of rows: who needs it, and when it is built anew."""
import types

import pytest


class FakeLibrary:
    """Takes every context and does nothing, so that no GPU is needed."""

    def wpsgd_create(self, device, stream, k, d, out):
        out._obj.value = 1
        return 0

    def wpsgd_destroy(self, h):
        return 0

    def wpsgd_launch_count(self, h):
        return 5


def test_a_context_needs_the_extension_for_these_operators_alone(monkeypatch):
    from paper_1708_04801_b200 import binding

    loads = []

    def load_rows():
        loads.append(1)
        raise RuntimeError("_rows.so is missing")

    monkeypatch.setattr(binding, "load_library", FakeLibrary)
    monkeypatch.setattr(binding, "load_rows", load_rows)
    with binding.Context(1, 4, device=0, stream=types.SimpleNamespace(cuda_stream=0)) as ctx:
        assert ctx.launch_count() == 5 and not loads
        for call in (lambda: ctx.quantize_rows(None), lambda: ctx.margins_fp8(None, None, None, None), lambda: ctx.objective_grad(None, None, None, 0.0, 0),
                     lambda: ctx.objective_grad_fp8(None, None, None, None, 0.0, 0)):
            with pytest.raises(RuntimeError, match="missing"):
                call()
        assert len(loads) == 4
        monkeypatch.setattr(binding, "load_rows", lambda: loads.append(1) or types.SimpleNamespace(quantize_rows=lambda *a: tuple(a)))
        assert ctx.quantize_rows("X") == (1, 0, 0, 4, "X", None, None)
        assert ctx.quantize_rows("Y")[4] == "Y" and len(loads) == 5   # loaded once


def test_the_extension_is_built_anew_for_another_torch(wpsgd_lib, monkeypatch):
    import torch

    from paper_1708_04801_b200 import binding, build

    assert build._binding_fresh()
    assert torch.__version__ in build._binding_stamp() and binding.load_rows().built_for == build._binding_stamp()
    monkeypatch.setattr(build, "_binding_stamp", lambda: "another torch")
    assert not build._binding_fresh()


def test_clipping_needs_a_norm_to_clip_to(monkeypatch):
    # the extension takes None for "the norm alone": a clip without a limit would return and leave the gradients as they are
    from paper_1708_04801_b200 import binding

    calls = []
    monkeypatch.setattr(binding, "load_library", FakeLibrary)
    monkeypatch.setattr(binding, "load_rows", lambda: types.SimpleNamespace(grad_norm=lambda *a: calls.append(a) or "norm"))
    monkeypatch.setattr(binding.Context, "_grad_list", lambda self, grads: types.SimpleNamespace(_h=types.SimpleNamespace(value=7)))
    with binding.Context(1, 4, device=0, stream=types.SimpleNamespace(cuda_stream=0)) as ctx:
        for limit in (None, "much", [1.0]):
            with pytest.raises((TypeError, ValueError)):
                ctx.clip_grad_norm([], limit)
        assert not calls
        assert ctx.clip_grad_norm([], 2) == "norm" and calls[0][4:] == (7, 2.0, None)
        assert ctx.grad_norm([]) == "norm" and calls[1][4:] == (7, None, None)
