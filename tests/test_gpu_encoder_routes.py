"""GPU tests of the encoder's products at the further sizes of encoder_shapes_more.py, with the checks of test_gpu_encoder.py and
test_gpu_encoder_tiles.py."""
import pytest

import test_gpu_encoder as small
import test_gpu_encoder_tiles as tiles
from encoder_shapes_more import FEW, MORE
from test_gpu_encoder import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def these_sizes(monkeypatch):
    monkeypatch.setattr(tiles, "TILES", MORE)
    monkeypatch.setattr(tiles, "TILES_8_BITS", MORE)
    monkeypatch.setattr(small, "SIZES", FEW)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(MORE)))
def test_linear_and_its_gradients(i, dtype):
    tiles.test_linear_and_its_gradients(i, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(MORE)))
def test_gated_and_its_gradients(i, dtype):
    tiles.test_gated_and_its_gradients(i, dtype)


@pytest.mark.parametrize("i", range(len(MORE)))
def test_products_of_8_bit_operands(i):
    tiles.test_products_of_8_bit_operands(i)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(FEW)))
def test_few_rows(i, dtype):
    small.test_linear_and_its_gradients(i, dtype)
    small.test_gated_and_its_gradients(i, dtype)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(FEW)))
def test_few_rows_of_8_bits(i, out_dtype):
    small.test_products_of_8_bit_operands(i, out_dtype)
