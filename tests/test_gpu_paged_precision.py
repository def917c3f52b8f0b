"""How exact pp_paged_attention's scores and probabilities are: float32's bits, whatever the pages hold and however large one
element of a query is."""
import math

import pytest
import torch

from paper_2404_09529_amd import prepack as pp

from .gpu_util import require_gpu
from .test_gpu_paged import KINDS, TYPES, U, Pool, check_attention, config, rand, run_attention

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


@pytest.mark.parametrize("table", ["narrow", "wide"])
@pytest.mark.parametrize("kv", ["bf16", "i8"])
def test_probabilities_that_nearly_cancel(kv, table):
    """Three keys: the likeliest with the value 0, and two of nearly equal probability with the values 1 and -1.  Scores
    are exact in float32.  x, a score's distance to the largest in powers of two, is off by 2^-23 of itself (its
    constant and its product are rounded), 2^x by that (times ln 2), a step of 2^-23 and what the terms leave, 2^-24; sums and
    products of three keys in three terms add 12 2^-24 of sum p |v|, and the result is rounded once."""
    k, H, D = 64, 16, 128
    pool = Pool(kv, k, 1, D, 16, 1 if table == "narrow" else 128, seed=1, spare=1)
    q = torch.zeros(k, H, D)
    g = torch.Generator().manual_seed(3)
    q[:, :, 0] = (0.5 + torch.rand(k, H, generator=g)).bfloat16().float()
    q[:, :, 1] = 2.0 ** -9
    for x in (pool.k, pool.v):
        x.zero_()
    if kv == "i8":
        pool.ks.fill_(1.0), pool.vs.fill_(1.0)
    keys, values = pool.k.view(-1, D), pool.v.view(-1, D)
    for i in range(k):
        a, b, m = (pool.row(i, j) for j in range(3))
        keys[m, 0] = 100
        keys[a, 0] = keys[b, 0] = 99 - i % 16
        keys[b, 1] = 1 + i // 16
        values[a], values[b] = 1, -1
    pool.to_device()
    got = run_attention(config(H, 1, D, "bf16"), pool, [3] * k, q.to(torch.bfloat16).view(k, -1).cuda())[:k].double().cpu().view(k, H, D)
    K, V = pool.values()
    rows = torch.tensor([[pool.row(i, j) for j in range(3)] for i in range(k)])
    s = (K[rows, 0][:, None] * q.double()[:, :, None]).sum(-1) / math.sqrt(D)      # [k, H, 3]
    p = torch.softmax(s, -1)
    want = (p[:, :, 0] - p[:, :, 1])[..., None].expand(k, H, D)
    x = (s.amax(-1) - s[..., 0]) / math.log(2)
    e = x * 2 * U + 2 * U + U
    tol = ((e + 12 * U) * (p[..., 0] + p[..., 1]))[..., None] + 2.0 ** -8 * want.abs()
    worst = float(((got - want).abs() / tol).max())
    print(f"[paged attention] worst error / tolerance {worst:.3f}", flush=True)
    assert worst <= 1.0
