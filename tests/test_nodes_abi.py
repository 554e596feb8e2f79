"""Rows sorted by node and back, and chains whose labels are vectors: what the C entries refuse before anything reaches a GPU."""
import ctypes


def test_null_contexts(wpsgd_lib):
    lib = wpsgd_lib
    assert lib.wpsgd_sort_rows(None, None, 1, 1, 1, None, None, None) == 1
    assert lib.wpsgd_gather_rows(None, None, 0, 1, 1, None, 1, 1, None, 1, 1) == 1
    assert lib.wpsgd_combine_rows(None, None, 0, 1, 1, 1, None, None, 1, 1, None, 1) == 1
    assert lib.wpsgd_combine_rows_grad(None, None, 1, None, 1, 0, 1, 1, None, None, 1, 1, None, 1, None) == 1
    assert lib.wpsgd_last_error(None) == b"ctx is NULL"


class DeltaRows(ctypes.Structure):
    """wpsgd_delta_rows"""

    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v", "g", "beta")] + [(n, ctypes.c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_g", "ld_beta")]
                + [("shard_off", ctypes.c_void_p), ("n_rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("n_chains", "heads_k", "heads_v", "dk", "dv")]
                + [("type", ctypes.c_int), ("scale", ctypes.c_float)])


RUN, SAVE, GRAD = 0, 1, 2


def rows(n=1000, chains=3, hk=2, hv=4, dk=64, dv=32, type=1):
    a = 1 << 20
    return DeltaRows(a, a, a, a, a, hk * dk, hk * dk, hv * dv, hv, hv, a, n, chains, hk, hv, dk, dv, type, 1.0)


def workspace(lib, r, use):
    n = ctypes.c_int64(-1)
    st = lib.wpsgd_delta_workspace(ctypes.byref(r) if r is not None else None, use, ctypes.byref(n))
    return st, n.value


def test_workspaces_of_chains(wpsgd_lib):
    st, run = workspace(wpsgd_lib, rows(), RUN)
    assert st == 0 and run > 0
    assert workspace(wpsgd_lib, rows(), SAVE)[1] > run and workspace(wpsgd_lib, rows(), GRAD)[1] > 0
    assert workspace(wpsgd_lib, rows(type=0), RUN) == (0, 0)                           # fp32 rows need none
    assert workspace(wpsgd_lib, rows(dk=60), RUN)[1] > run                             # heads that are laid out anew
    assert workspace(wpsgd_lib, rows(n=1 << 20, chains=1, hv=32), SAVE)[1] > 1 << 32   # sizes pass 32 bits
    assert workspace(wpsgd_lib, rows(n=0, chains=0), GRAD)[0] == 0


def test_chains_that_are_refused(wpsgd_lib):
    lib = wpsgd_lib
    for r, status in ((None, 1), (rows(n=-1), 1), (rows(chains=-1), 1), (rows(hk=0), 1), (rows(hk=3), 1), (rows(dv=0), 1), (rows(type=2), 1), (rows(dk=129), 5), (rows(dv=200), 5),
                      (rows(n=1 << 40), 5), (rows(chains=1 << 30), 5)):
        assert workspace(lib, r, RUN) == (status, 0)
        assert lib.wpsgd_last_error(None).startswith(b"delta_workspace:")
    assert workspace(lib, rows(), 3)[0] == 1 and workspace(lib, rows(type=0), SAVE)[0] == 5 and workspace(lib, rows(type=0), GRAD)[0] == 5
    assert lib.wpsgd_delta_workspace(ctypes.byref(rows()), RUN, None) == 1
    assert lib.wpsgd_delta_run(None, None, None, None, None, 1, RUN, None, 0) == 1
    assert lib.wpsgd_delta_grad(None, None, None, 0, None, 1, None, None, None, None, None, None, None, None, 0) == 1
    assert lib.wpsgd_delta_step(None, None, None, None, 1, None, 1) == 1
