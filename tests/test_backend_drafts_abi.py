"""The C-ABI of the operators for drafts and beams without a GPU: record layouts, calls without a handle, what is refused before any CUDA call."""
import ctypes as C

from paper_2603_20661_b200 import backend
from paper_2603_20661_b200 import build as cuda_build


def lib():
    cuda_build.build()
    return backend._lib()


def test_struct_layouts_match_the_header():
    assert C.sizeof(backend.RotationRecord) == 4 * 8 + 4 * 4 and C.sizeof(backend.ForkRecord) == 10 * 8 + 2 * 4


def test_calls_without_a_handle_are_refused():
    b = lib()
    assert b.wwws_attend_tree(None, None, None, None, 0, None, 0, 1.0, 0, 0, None, 0) == 1
    assert b.wwws_rotate(None, None, 0, None, None, 0, None, 0, None, 0, None, 0) == 1
    assert b.wwws_rotate_append(None, None, None, None, None, None, 0, None, 0, None, 0, None, 0) == 1
    assert b.wwws_pages_fork(None, None) == 1 and b.wwws_cache_copy(None, None, 0, None, 0) == 1 and b.wwws_cache_compact(None, None, None, 0, None, None, 0) == 1
    assert b.wwws_select_beams(None, 0, 1, 1, 0, None, 1, None, 1, None, 0, None, None, None) == 1


def test_scratch_of_the_beams():
    b, n = lib(), C.c_uint64()
    for good in ((1, 1, 0, 1), (65535, 32000, 2, 8), (64, 1 << 24, 1, 128), (0, 5, 0, 1)):
        assert b.wwws_beams_scratch_bytes(*good, C.byref(n)) == 0
        assert (n.value > 0) == (good[0] > 0) and n.value % 8 == 0
    for bad in ((65536, 5, 0, 1), (1, 0, 0, 1), (1, (1 << 24) + 1, 0, 1), (1, 5, 3, 1), (1, 5, 0, 0), (1, 5, 0, 129)):
        assert b.wwws_beams_scratch_bytes(*bad, C.byref(n)) == 1
        assert len(b.wwws_backend_last_error(None)) > 0
    assert b.wwws_beams_scratch_bytes(1, 5, 0, 1, None) == 1


def test_a_turn_has_the_digits_that_its_64_bits_need():
    """Far positions multiply the error of a frequency in turns: against a series of 2 pi in whole numbers (Machin's formula)."""
    def arctan(x, one):                                      # of 1 / x
        total, term, n, sign = 0, one // x, 1, 1
        while term:
            total, term, n, sign = total + sign * (term // n), term // (x * x), n + 2, -sign
        return total
    one = 10 ** 60
    tau = 2 * 4 * (4 * arctan(5, one) - arctan(239, one))
    assert abs(backend.TAU * one - tau) < 10 ** 22
