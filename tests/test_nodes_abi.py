"""Rows sorted by node and back: what the C entries refuse before anything reaches a GPU."""


def test_null_contexts(wpsgd_lib):
    lib = wpsgd_lib
    assert lib.wpsgd_sort_rows(None, None, 1, 1, 1, None, None, None) == 1
    assert lib.wpsgd_gather_rows(None, None, 0, 1, 1, None, 1, 1, None, 1, 1) == 1
    assert lib.wpsgd_combine_rows(None, None, 0, 1, 1, 1, None, None, 1, 1, None, 1) == 1
    assert lib.wpsgd_combine_rows_grad(None, None, 1, None, 1, 0, 1, 1, None, None, 1, 1, None, 1, None) == 1
    assert lib.wpsgd_last_error(None) == b"ctx is NULL"
