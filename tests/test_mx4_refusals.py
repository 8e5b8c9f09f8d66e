"""Microscaled 4-bit rows without a GPU: the reference's own rules, and what the binding refuses before it calls the library."""
import numpy as np
import pytest

from tests import mx4_reference as R

torch = pytest.importorskip("torch")


def test_reference_rounds_to_nearest_ties_to_even():
    x = np.array([[4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, -0.3, -0.0, 0.2499, 0.2501] + [0.0] * 19])
    codes, scales = R.quantize(x)
    assert scales.tolist() == [[127]]
    want = [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -0.5, -0.0, 0.0, 0.5] + [0.0] * 19
    got = R.values(codes, scales, 32)[0]
    assert got.tolist() == want and np.signbit(got[10])


def test_reference_scales():
    x = np.zeros((1, 200))
    x[0, 32], x[0, 64], x[0, 96], x[0, 128], x[0, 160] = 1.0, np.inf, 2.0 ** -140, 3.9, np.nan
    assert R.quantize(x)[1].tolist() == [[0, 125, 255, 0, 126, 255, 0]]


@pytest.mark.parametrize("dim", [1, 31, 32, 33, 100])
def test_reference_keeps_stored_values(dim):
    """Values that rows of this form stand for come back the same (a block's scale is its own again or finer)."""
    rng = np.random.default_rng(dim)
    x = R.values(*R.quantize(rng.standard_normal((50, dim))), dim)
    assert np.array_equal(R.values(*R.quantize(x), dim), x)


def test_binding_refuses_what_is_not_rows_of_this_form():
    from paper_1305_1422_amd import capi
    host = torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    with pytest.raises(TypeError):
        capi._mx4(*host, "the")                              # host memory
    with pytest.raises(TypeError):
        capi._typed(torch.zeros(4, 32), "rows")


def test_library_refuses_calls_without_a_context():
    from paper_1305_1422_amd import capi
    L = capi.load()
    assert L.som_mx4_quantize(None, None, 0, 1, 1, None, None) == capi.SOM_ERR_INVALID_ARG
    assert L.som_mx4_dequantize(None, None, None, 1, None, 0, 1) == capi.SOM_ERR_INVALID_ARG
    assert L.som_mx4_product(None, None, None, 1, None, None, 1, None, 0, 1) == capi.SOM_ERR_INVALID_ARG
    assert L.som_bmus_mx4(None, None, None, 1, None, None, None) == capi.SOM_ERR_INVALID_ARG
    assert L.som_update_mx4(None, None, None, 1, None, None, 1.0, 1.0) == capi.SOM_ERR_INVALID_ARG
    assert L.som_train_epoch_mx4(None, None, None, 1, None, 1.0, 1.0, None) == capi.SOM_ERR_INVALID_ARG
    assert L.som_set_data_mx4(None, None, None, 1) == capi.SOM_ERR_INVALID_ARG


def test_mx4_is_not_taken_for_a_csr_triple():
    from paper_1305_1422_amd import som
    data = som.Mx4(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8))
    assert som._is_mx4(data) and not som._is_csr(data)
