"""Rows by node and chains whose labels are vectors: what their Python calls pass on and return, without a GPU."""
import types

import pytest


class FakeLibrary:
    """Takes every context and does nothing."""

    def wpsgd_create(self, device, stream, k, d, out):
        out._obj.value = 1
        return 0

    def wpsgd_destroy(self, h):
        return 0

    def wpsgd_last_error(self, h):
        return b"why"


def test_chains_and_nodes_go_through_the_extension(monkeypatch):
    from paper_1708_04801_b200 import binding

    calls = []
    monkeypatch.setattr(binding, "load_library", FakeLibrary)
    fake = types.SimpleNamespace(sort_rows=lambda *a: calls.append(a) or ("where", "order", "off"), delta_run=lambda *a: calls.append(a) or ("out", "W", "kept" if a[-1] else None),
                                 delta_grad=lambda *a: calls.append(a) or (1, 2, 3, 4, 5, None), delta_step=lambda *a: calls.append(a) or "out",
                                 gather_rows=lambda *a: 1)
    monkeypatch.setattr(binding, "load_rows", lambda: fake)
    with binding.Context(3, 4, device=0, stream=types.SimpleNamespace(cuda_stream=0)) as ctx:
        assert ctx.sort_rows("node") == ("where", "order", "off") and calls[-1][4:] == ("node", 3)
        assert ctx.delta_run("q", "k", "v", "g", "b", "off") == ("out", "W") and calls[-1][4:] == ("q", "k", "v", "g", "b", None, "off", None, None, None, False)
        out, W, saved = ctx.delta_run("q", "k", "v", "g", "b", "off", scale=2.0, save=True)
        assert saved.args == ("q", "k", "v", "g", "b", 2.0, "off", "kept")
        assert ctx.delta_grad(saved, "dout")[5] is None and calls[-1][4:] == saved.args + ("dout", None, False)
        assert ctx.delta_step("q", "k", "v", "g", "b", "W", "slots") == "out" and calls[-1][4:] == ("q", "k", "v", "g", "b", None, "W", "slots", None)
        with pytest.raises(binding.WpsgdError, match="wpsgd_gather_rows: WPSGD_ERR_INVALID_ARG: why"):
            ctx.gather_rows("X", "where")
