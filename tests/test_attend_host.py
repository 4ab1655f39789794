"""Host-side refusals of attention over shared pages, of page sharing and of their selectors: before any device work."""
import ctypes as C

import pytest

import paper_2510_01336_amd as hs


@pytest.fixture(scope="module")
def lib():
    lib = C.CDLL(hs.lib_path())
    lib.ee_last_error.restype = C.c_char_p
    lib.ee_rules_bytes.restype = C.c_size_t
    return lib


def test_null_arguments(lib):
    ints = (C.c_int32 * 4)()
    calls = [("ee_prefill_shared", (None, ints, ints, ints, ints)), ("ee_attend_begin", (None, ints, ints)),
             ("ee_attend", (None, 0, None, 1, C.c_int64(0), None, C.c_int64(0))), ("ee_rules_set", (None, 0, None)),
             ("ee_rules_rows", (None, 0, 0, None)), ("ee_rules_attach", (None, 0, None, C.c_size_t(0))), ("ee_logit_rules", (None, None))]
    for name, args in calls:
        assert getattr(lib, name)(*args) == -1, name
        assert lib.ee_last_error(), name
    assert lib.ee_shared_pages(None, 0) == -1
    assert lib.ee_rules_bytes(None, 0) == 0


def test_selectors_check_their_arguments(lib):
    for ok in (0, 1, -1):
        assert lib.ee_debug_shared_attention(ok) == 0, ok
    for bad in (-2, 2):
        assert lib.ee_debug_shared_attention(bad) == -1 and lib.ee_last_error(), bad
    for ok in (0, 100, -1):
        assert lib.ee_debug_rules_looks(ok) == 0, ok
    assert lib.ee_debug_rules_looks(-2) == -1 and lib.ee_last_error()
