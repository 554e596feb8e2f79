"""Operators on whole sets of rows: what they refuse, as far as no GPU is needed for it."""
import ctypes

import numpy as np
import pytest


def make(lib, grads, outs, sizes, types):
    n = len(sizes)
    g = np.array(grads, dtype=np.uint64)
    o = None if outs is None else np.array(outs, dtype=np.uint64)
    s, t = np.array(sizes, dtype=np.int64), np.array(types, dtype=np.int32)
    h = ctypes.c_void_p()
    st = lib.wpsgd_grad_list_create(g.ctypes.data, None if o is None else o.ctypes.data, s.ctypes.data, t.ctypes.data, n, ctypes.byref(h))
    if h.value:
        assert lib.wpsgd_grad_list_destroy(h) == 0
    assert (st == 0) == bool(h.value)
    return st


A = 1 << 20  # an address; lists are only checked here, never followed


@pytest.mark.parametrize("grads,outs,sizes,types", [
    ([A], None, [100], [0]),
    ([A, A + 400], None, [100, 100], [0, 0]),                      # one behind the other
    ([A, A], [A + 1000, A + 2000], [100, 100], [0, 0]),            # one input twice, outputs apart
    ([A, A + 400], [A, A + 8000], [100, 100], [0, 0]),             # in place and apart in one list
    ([0, A], None, [0, 4], [0, 1]),                                # a tensor without elements has no address
    ([A + 2], None, [3], [1]),
])
def test_lists_that_are_taken(wpsgd_lib, grads, outs, sizes, types):
    assert make(wpsgd_lib, grads, outs, sizes, types) == 0


@pytest.mark.parametrize("grads,outs,sizes,types", [
    ([A, A], None, [100, 100], [0, 0]),                            # the same tensor twice, in place
    ([A, A + 396], None, [100, 100], [0, 0]),                      # one element shared
    ([A], [A + 4], [100], [0]),                                    # shifted onto itself
    ([A, A + 4000], [A + 4000, A + 8000], [100, 100], [0, 0]),     # one's output is another's input
    ([A, A + 4000], [A + 8000, A + 8100], [100, 100], [0, 0]),     # outputs overlap
    ([A + 2], None, [3], [0]),                                     # fp32 off its alignment
    ([A + 1], None, [3], [1]),
    ([A], [A + 1001], [3], [1]),
    ([0], None, [1], [0]),
    ([A], [0], [1], [0]),
    ([A], None, [-1], [0]),
    ([A], None, [1 << 50], [0]),
    ([A], None, [1], [2]),
])
def test_lists_that_are_refused(wpsgd_lib, grads, outs, sizes, types):
    assert make(wpsgd_lib, grads, outs, sizes, types) == 1
    assert wpsgd_lib.wpsgd_last_error(None).startswith(b"grad_list_create:")


def test_null_arguments(wpsgd_lib):
    lib = wpsgd_lib
    h = ctypes.c_void_p()
    assert lib.wpsgd_grad_list_create(None, None, None, None, 1, ctypes.byref(h)) == 1
    assert lib.wpsgd_grad_list_create(None, None, None, None, 0, None) == 1
    assert lib.wpsgd_grad_list_create(None, None, None, None, -1, ctypes.byref(h)) == 1
    assert lib.wpsgd_grad_list_create(None, None, None, None, 0, ctypes.byref(h)) == 0 and h.value
    assert lib.wpsgd_grad_list_destroy(h) == 0 and lib.wpsgd_grad_list_destroy(None) == 0
    assert lib.wpsgd_quantize_rows(None, None, 0, 1, 1, None, 16, None, 1) == 1
    assert lib.wpsgd_margins_fp8(None, None, 16, None, 1, 1, None, 16, None, 1, 1, None, 0, 1) == 1
    assert lib.wpsgd_objective_grad(None, None, 0, 1, None, 1, None, 0.0, 0, None, None) == 1
    assert lib.wpsgd_objective_grad_fp8(None, None, 16, None, 1, None, 1, None, 0.0, 0, None, None) == 1
    assert lib.wpsgd_grad_norm(None, None, None) == 1
    assert lib.wpsgd_clip_grad_norm(None, None, 1.0, None) == 1


def test_binding_refuses_what_it_can_see(wpsgd_lib):
    import torch

    import paper_1708_04801_b200 as P

    with pytest.raises(TypeError):
        P.GradList([torch.zeros(3)])          # not on a GPU
    with pytest.raises(ValueError):
        P.GradList([torch.zeros(3)], [])
    assert P.packed_width(1) == 16 and P.packed_width(16) == 16 and P.packed_width(999) == 1008
