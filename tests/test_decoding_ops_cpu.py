"""What the decoding operators' C entries refuse, on the host alone: no call here reaches the device."""
import ctypes as C

import pytest
import torch

from paper_1802_07170_amd import binding, decoding

E = binding.CMT_EINVAL
AT = 1 << 20                                                 # an address that is never used


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def text(lib):
    return lib.cmt_operator_error().decode()


def test_sizes(lib):
    n = C.c_size_t()
    assert lib.cmt_quant_weight_bytes(32000, 1024, 64, C.byref(n)) == 0
    assert n.value == 32000 * 512 + 32000 * 16 * 2
    assert lib.cmt_quant_weight_bytes(1, 1, 32, C.byref(n)) == 0 and n.value % 256 == 0 and n.value >= 1024
    assert lib.cmt_cache_bytes(C.byref(binding.CmtCacheConfig(64, 1, 1024, 50)), C.byref(n)) == 0
    assert n.value == 256 + 2 * 512 + 2 * 64 * 64 * 1024
    assert lib.cmt_beam_select_workspace(64, 10, 32000, C.byref(n)) == 0 and n.value == 640 * 63 * 8
    for args in ((0, 5, 32), (5, 0, 32), (5, 5, 48), (1 << 25, 5, 32), (5, 1 << 17, 32), (1 << 22, 1 << 15, 32)):
        assert lib.cmt_quant_weight_bytes(*args, C.byref(n)) == E, args
    for args in ((0, 1, 8, 8), (1, 0, 8, 8), (1, 1, 0, 8), (1, 1, 1025, 8), (1, 1, 8, 0), (70000, 1, 8, 8)):
        assert lib.cmt_cache_bytes(C.byref(binding.CmtCacheConfig(*args)), C.byref(n)) == E, args
    for args in ((0, 1, 8), (1, 0, 8), (1, 33, 8), (1, 1, 0), (1, 1, 1 << 27)):
        assert lib.cmt_beam_select_workspace(*args, C.byref(n)) == E, args
    assert lib.cmt_quant_weight_bytes(5, 5, 32, None) == E and text(lib) == "null pointer"


def test_the_product_s_arguments(lib):
    good = [AT, 1, 64, 3, AT, 20, 64, 32, None, 0, AT, 0, 20, None]
    for at, bad in ((0, None), (0, AT + 1), (1, 2), (2, 63), (3, -1), (3, 70000), (4, None), (4, AT + 16), (5, 0), (7, 31), (8, AT + 2), (10, None), (10, AT + 2),
                    (11, 3), (12, 19)):
        args = list(good)
        args[at] = bad
        assert lib.cmt_quant_product(*args) == E, (at, bad)
        assert text(lib)
    good[3] = 0
    assert lib.cmt_quant_product(*good) == 0                 # no rows: nothing is done
    for args in ((None, 0, 64, 20, 64, 32, AT, None), (AT, 0, 63, 20, 64, 32, AT, None), (AT, 5, 64, 20, 64, 32, AT, None), (AT, 0, 64, 20, 64, 32, AT + 8, None)):
        assert lib.cmt_quant_weight_pack(*args) == E, args
    assert lib.cmt_quant_weight_encode(AT, None, 20, 64, 32, AT, None) == E
    assert lib.cmt_quant_weight_values(AT, 20, 64, 32, AT + 1, None) == E


def test_the_cache_s_arguments(lib):
    cfg = binding.CmtCacheConfig(2, 2, 64, 500)
    rows = lambda *s: C.byref(binding.CmtCacheRows(AT, *s))
    for args in ((None, rows(1, 1, 1), rows(1, 1, 1), 0, AT, 5), (AT, None, rows(1, 1, 1), 0, AT, 5), (AT, rows(1, 1, 1), rows(1, 1, 1), 0, None, 5),
                 (AT, rows(1, 1, 1), rows(1, 1, 1), 7, AT, 5), (AT, rows(1, 1, 1), rows(1, 1, 1), 0, AT, 501), (AT, rows(1, 1, 1), rows(1, 1, 1), 0, AT, 0),
                 (AT, rows(1, 1, 1), rows(1, -1, 1), 0, AT, 5), (AT + 4, rows(1, 1, 1), rows(1, 1, 1), 0, AT, 5)):
        assert lib.cmt_cache_fill(C.byref(cfg), *args, None) == E, args
    need = C.c_size_t()
    assert lib.cmt_cache_attend_workspace(C.byref(cfg), 3, 4, 500, C.byref(need)) == 0 and need.value > 0
    good = [AT, AT, 1, 256, 3, 4, 500, 1.0, AT, 256, AT, need.value, None]
    for at, bad in ((0, None), (1, None), (2, 4), (3, 255), (4, 0), (5, 3), (5, 0), (6, 0), (6, 501), (7, float("nan")), (8, None), (9, 255), (10, None), (10, AT + 8),
                    (11, need.value - 1)):
        args = list(good)
        args[at] = bad
        assert lib.cmt_cache_attend(C.byref(cfg), *args) == E, (at, bad)
    assert lib.cmt_cache_attend_workspace(C.byref(cfg), 3, 4, 100, C.byref(need)) == 0 and need.value == 0     # one range: no parts to join
    assert lib.cmt_cache_read(C.byref(cfg), AT, 501, AT, AT, None) == E


def test_the_search_s_arguments(lib):
    need = C.c_size_t()
    assert lib.cmt_beam_select_workspace(2, 3, 1000, C.byref(need)) == 0
    good = [AT, 1, 1000, AT, 2, 3, 1000, 3, AT, AT, AT, AT, need.value, None]
    for at, bad in ((0, None), (0, AT + 1), (1, 9), (2, 999), (3, None), (4, 0), (5, 33), (6, 0), (7, 0), (7, 33), (8, None), (9, AT + 2), (10, None), (11, None),
                    (12, need.value - 1)):
        args = list(good)
        args[at] = bad
        assert lib.cmt_beam_select(*args) == E, (at, bad)
    one = lambda *a: (binding.CmtReorderTensor * 1)(binding.CmtReorderTensor(*a))
    for job in (one(None, AT, 8, 8, 8), one(AT, None, 8, 8, 8), one(AT, 2 * AT, 7, 8, 8), one(AT, 2 * AT, 8, 7, 8), one(AT, 2 * AT, 8, 8, 0), one(AT, AT + 8, 8, 8, 8)):
        assert lib.cmt_beam_reorder(AT, 4, 4, job, 1, None) == E
    fine = one(AT, 2 * AT, 8, 8, 8)
    assert lib.cmt_beam_reorder(None, 4, 4, fine, 1, None) == E and lib.cmt_beam_reorder(AT, -1, 4, fine, 1, None) == E
    assert lib.cmt_beam_reorder(AT, 4, 4, fine, 257, None) == E and "256" in text(lib)
    assert lib.cmt_beam_reorder(AT, 0, 4, fine, 1, None) == 0 and lib.cmt_beam_reorder(AT, 4, 4, None, 0, None) == 0


def test_tensors_off_the_device_are_refused():
    x = torch.zeros(2, 64)
    for call in (lambda: decoding.QuantWeight.pack(x), lambda: decoding.beam_select(x, torch.zeros(2, 1)),
                 lambda: decoding.beam_reorder(torch.zeros(2, dtype=torch.int32), [x], [x])):
        with pytest.raises(ValueError):
            call()


def test_more_than_a_launch_can_count(lib):
    """Grids of 2^32 threads and more are refused as arguments, not by the launch."""
    n = C.c_size_t()
    assert lib.cmt_quant_weight_bytes(1 << 18, 1 << 16, 64, C.byref(n)) == 0
    assert lib.cmt_quant_weight_bytes((1 << 18) + 1, 1 << 16, 64, C.byref(n)) == E and "2^34" in text(lib)
    assert lib.cmt_quant_product(AT, 1, 64, 65535, AT, 1 << 21, 64, 32, None, 0, AT, 0, 1 << 21, None) == E and "2^36" in text(lib)
    assert lib.cmt_beam_select_workspace(1 << 10, 32, 1 << 19, C.byref(n)) == 0
    assert lib.cmt_beam_select_workspace(1 << 10, 32, (1 << 19) + 1, C.byref(n)) == E and "2^25" in text(lib)
    job = (binding.CmtReorderTensor * 1)(binding.CmtReorderTensor(AT, 1 << 40, 8, 8, 8))
    assert lib.cmt_beam_reorder(AT, (1 << 24) + 1, 4, job, 1, None) == E and "2^24" in text(lib)


def test_a_target_on_the_rows_numbers_is_refused(lib):
    job = lambda at: (binding.CmtReorderTensor * 1)(binding.CmtReorderTensor(AT, at, 8, 8, 8))
    for at in (2 * AT, 2 * AT + 12, 2 * AT - 24):
        assert lib.cmt_beam_reorder(2 * AT, 4, 4, job(at), 1, None) == E and "numbers" in text(lib), at
