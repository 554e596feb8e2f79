"""Rows that a call leaves out: what the C entries refuse before anything reaches a GPU."""


def test_null_contexts(wpsgd_lib):
    assert wpsgd_lib.wpsgd_clear_rows(None, None, 1, 1, None, 0, 1, 1, 1, None) == 1
    assert wpsgd_lib.wpsgd_last_error(None) == b"ctx is NULL"
