"""Sizes, windows and numbers that the C structs cannot hold are refused by the
binding, not cut off on the way."""
import pytest

from paper_2602_01219_amd import mita


@pytest.mark.parametrize("field", ["B", "H", "N", "d", "H_kv", "N_k"])
@pytest.mark.parametrize("value", [2 ** 32 + 64, 2 ** 31, -2 ** 33])
def test_dense_sizes(field, value):
    kw = dict(B=2, H=4, N=8, d=64)
    kw[field] = value
    with pytest.raises(ValueError, match=field):
        mita.DenseConfig(**kw).struct()


@pytest.mark.parametrize("field", ["left", "right"])
@pytest.mark.parametrize("value", [2 ** 32, 2 ** 32 + 5, 2 ** 32 - 1, 2 ** 31, -2 ** 31 - 1])
def test_dense_windows(field, value):
    with pytest.raises(ValueError, match=field):
        mita.DenseConfig(2, 4, 8, 64, **{field: value}).struct()
    assert getattr(mita.DenseConfig(2, 4, 8, 64, **{field: 2 ** 31 - 1}).struct(), field) == 2 ** 31 - 1


@pytest.mark.parametrize("rows", [(2 ** 32 + 5,), (3, 2 ** 32), (2 ** 31, 1, 1)])
def test_norm_rows(rows):
    with pytest.raises(ValueError, match="rows"):
        mita.NormConfig(rows, 64).struct()


def test_norm_width():
    with pytest.raises(ValueError, match="C"):
        mita.NormConfig((4,), 2 ** 32 + 64).struct()


def test_numbers_that_fp32_rounds_to_zero():
    # a scale of 0 means 1 / sqrt(d)
    with pytest.raises(ValueError, match="scale"):
        mita.DenseConfig(2, 4, 8, 64, scale=1e-60).struct()
    with pytest.raises(ValueError, match="eps"):
        mita.NormConfig((4,), 64, eps=1e-60).struct()
    assert mita.DenseConfig(2, 4, 8, 64, scale=0.0).struct().scale == 0.0
