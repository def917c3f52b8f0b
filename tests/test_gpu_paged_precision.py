"""How exact pp_paged_attention's scores are: float32's bits, whatever the pages hold and however large one element of a
query is."""
import pytest
import torch

from paper_2404_09529_amd import prepack as pp

from .gpu_util import require_gpu
from .test_gpu_paged import KINDS, TYPES, Pool, check_attention, config, rand, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("loud", [2.0 ** 10, 2.0 ** 20])
@pytest.mark.parametrize("lens", [[600, 33, 1, 300], [5000, 33, 1, 300]])
@pytest.mark.parametrize("dtype,kv", KINDS)
def test_loud_elements_of_a_query(dtype, kv, lens, loud):
    """Elements far above the others, which the keys do not have: they add nothing, and the others keep their bits."""
    H, Hkv, D = (8, 2, 128) if dtype == "bf16" else (8, 2, 64)
    pool = Pool(kv, len(lens), Hkv, D, 16, -(-max(lens) // 16), seed=5).fill(6)
    pool.k.view(-1, Hkv, D)[:, :, [7, 40]] = 0
    pool.to_device()
    q = 2.0 * rand(torch.Generator().manual_seed(8), len(lens), H, D)
    q[:, ::2, 7], q[:, 1::2, 40] = loud, -1.375 * loud
    q = q.to(TYPES[dtype][1])
    got = run_attention(config(H, Hkv, D, dtype), pool, lens, q.view(len(lens), -1).cuda())
    check_attention(got, q.double(), pool, lens, H, dtype)
