"""pp_quantize_rows, pp_dequantize_rows and pp_rmsnorm_quant at a length just below each at which another kernel
takes the rows."""
import pytest
import torch

from paper_2404_09529_amd import prepack as pp

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


@pytest.mark.parametrize("rows,d", [(3, 16400), (2, 400016), (2, 4000016), (1, 40000016)])
@pytest.mark.parametrize("value", [1.0002, None])
def test_norm_of_dense_long_rows(rows, d, value):
    """The sum of many squares of one size.  Equal values are the worst: additions of a float32 to a float32 sum
    all round the same way.  A square and two additions of four are off by 3 U, the mean by U and the sum with eps by
    U: 2.5 U after the root, itself 2 U, and two products 2 U."""
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.full((rows, d), value, device="cuda") if value else torch.randn((rows, d), generator=g, device="cuda")
    gain = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    y = x.double() / (x.double().square().mean(dim=1, keepdim=True) + 1e-5).sqrt() * gain.double()
    q, scale = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    pp.pp_rmsnorm_quant(pp.PP_F32, x, None, gain, rows, d, 1e-5, q, scale)
    top = y.abs().amax(dim=1)
    rel = 6.6 * G.U
    assert bool(((scale.double() * 127 - top).abs() <= (rel + 2.01 * G.U) * top).all())
    t = y / scale.double()[:, None]
    assert bool(((q.double() - t).abs() <= 0.5 + 127.1 * (2 * G.U + 2 * rel)).all())
