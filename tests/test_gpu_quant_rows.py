"""pp_quantize_rows, pp_dequantize_rows and pp_rmsnorm_quant at a length just below each at which another kernel
takes the rows."""
import pytest

from . import test_gpu_quant as G
from .gpu_util import require_gpu

pytestmark = pytest.mark.gpu

LENGTHS = [240, 400, 1008, 2032, 4080, 6128, 8176, 11008, 16368, 32752, 65520, 131056, 131088]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("d", LENGTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_in_8_bits_and_back(d, dtype):
    G.test_quantize_rows(5, d, dtype)
    G.test_dequantize_rows(5, d, dtype)


@pytest.mark.parametrize("d", LENGTHS)
@pytest.mark.parametrize("add", [None, "bf16", "f32"])
def test_norm(d, add):
    G.test_rmsnorm_quant(5, d, add)
