"""Refusals of the acoustic-model operators, of the library and of its binding
(no GPU needed: the checks come before any device call)."""
import pytest

from test_am_abi import MAKE, am, put  # noqa: F401

torch = pytest.importorskip("torch")


def refused(am, name, **change):  # noqa: F811
    from paper_1808_00687_amd import wfstdec
    a = MAKE[name](am)
    for path, v in change.items():
        put(a, path.replace("__", "."), v)
    return (getattr(am._lib, "wfst_am_" + name)(bytes(a), None) == wfstdec.WFST_EINVAL
            and wfstdec.wfst_last_error().startswith("wfst_am_" + name))


@pytest.mark.parametrize("value", [-1, 2])
def test_round_dz_is_zero_or_one(am, value):  # noqa: F811
    assert refused(am, "linear_backward", round_dz=value)


@pytest.mark.parametrize("name", ["distill", "distill_backward"])
def test_temperature_has_a_reciprocal(am, name):  # noqa: F811
    assert refused(am, name, temperature=2.0 ** -127)


def test_products_of_more_elements_than_any_memory(am):  # noqa: F811
    for change in ({"x__rows": 1 << 30, "y__rows": 1 << 30, "w__rows": 1 << 11, "y__cols": 1 << 11, "y__row_stride": 1 << 11},
                   {"w__rows": 1 << 30, "x__rows": 1 << 11, "y__rows": 1 << 11, "y__cols": 1 << 30, "y__row_stride": 1 << 30}):
        assert refused(am, "linear", residual__data=None, pre__data=None, **change)
        from paper_1808_00687_amd import wfstdec
        assert "2^40" in wfstdec.wfst_last_error()


def test_slices_that_share_a_column(am):  # noqa: F811
    # x [4 x 16], w, residual, pre and y [4 x 8], rows 64 values apart in one buffer of 4-byte values
    at = 0x10000000
    for y, pre in ((0, 7), (7, 0), (0, -7), (60, 0), (0, 60), (0, 64 + 7), (0, 64 - 7), (0, 3 * 64 + 1)):
        assert refused(am, "linear", y__data=at + 4 * y + 4096, y__row_stride=64, pre__data=at + 4 * pre + 4096, pre__row_stride=64)
    # another stride: by the whole spans
    assert refused(am, "linear", y__data=at + 4096, y__row_stride=64, pre__data=at + 4096 + 32, pre__row_stride=128)
