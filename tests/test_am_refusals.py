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
