"""Every way that pp_gemm_quant may go through its kernels, one size each, against float64.

``tests/test_quant_choice.py`` asks the library's own choice, on the CPU, whether these sizes still go the
ways they are named for."""
import pytest
import torch

from paper_2404_09529_amd import prepack as pp

from .gpu_util import require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": (pp.PP_BF16, torch.bfloat16), "f32": (pp.PP_F32, torch.float32)}

# Rows as they are: way -> (M, N, K).  ("few", column blocks, row blocks), ("tile", rows x columns, shares
# of K, whether 256 x 256 tiles go before), or the tile of the large kernel.
ROWS = {
    ("few", 1, 1): (1, 544, 144), ("few", 1, 2): (17, 32, 16), ("few", 1, 4): (33, 32, 16), ("few", 2, 1): (1, 4128, 16),
    ("few", 2, 2): (17, 4128, 16), ("few", 2, 4): (33, 4288, 16), ("few", 4, 1): (1, 8224, 16),
    ("tile", "32x64", 1, False): (65, 32, 16), ("tile", "32x64", 2, False): (1, 4288, 16368),
    ("tile", "32x64", 3, False): (1, 4160, 17712), ("tile", "32x64", 4, False): (33, 32, 5360),
    ("tile", "32x64", 6, False): (17, 32, 9360), ("tile", "32x64", 8, False): (1, 32, 15920),
    ("tile", "64x64", 1, False): (8194, 32, 16), ("tile", "64x64", 2, False): (5435, 32, 11184),
    ("tile", "64x64", 3, False): (4126, 32, 7728), ("tile", "64x64", 4, False): (2786, 32, 6576),
    ("tile", "64x64", 6, False): (2060, 32, 11216), ("tile", "64x64", 8, False): (1346, 32, 19088),
    ("tile", "64x128", 1, False): (67, 10976, 16), ("tile", "64x128", 2, False): (35, 8544, 10896),
    ("tile", "64x128", 3, False): (33, 5472, 11664), ("tile", "64x128", 4, False): (69, 2752, 9136),
    ("tile", "64x128", 6, False): (65, 2208, 11600), ("tile", "64x128", 8, False): (69, 1856, 16976),
    ("tile", "128x128", 1, False): (65, 22208, 16), ("tile", "128x128", 2, False): (8288, 32, 11344),
    ("tile", "128x128", 3, False): (66, 6112, 8080), ("tile", "128x128", 4, False): (67, 5632, 7344),
    ("tile", "128x128", 6, False): (69, 2752, 11376), ("tile", "128x128", 8, False): (71, 2784, 12112),
    ("tile", "128x256", 1, False): (196, 25408, 16),
    ("tile", "32x64", 1, True): (538, 22688, 144), ("tile", "64x64", 1, True): (1315, 10880, 144),
    ("tile", "64x128", 1, True): (565, 22048, 144), ("tile", "128x128", 1, True): (579, 26496, 144),
    ("tile", "128x256", 1, True): (1165, 28704, 1648),
    ("192x192",): (264, 21952, 144), ("192x256",): (385, 17024, 144), ("256x256",): (403, 22112, 144)}

# Over a plan of `rows` prompts of `length` tokens, a row of `capacity` each: way, and whether the list names
# every row tile -> (rows, capacity, length, N, K).
LISTS = {
    ("tile", "32x64", 1, False, False): (1, 265, 147, 32, 144), ("tile", "32x64", 1, False, True): (1, 257, 257, 32, 144),
    ("tile", "64x64", 1, False, False): (6, 1412, 1217, 32, 144), ("tile", "64x64", 1, False, True): (13, 631, 631, 32, 144),
    ("tile", "64x128", 1, False, False): (14, 604, 411, 96, 144), ("tile", "64x128", 1, False, True): (16, 513, 513, 96, 144),
    ("tile", "128x128", 1, False, False): (24, 459, 419, 160, 144),
    ("tile", "128x128", 1, False, True): (18, 605, 605, 160, 144),
    ("tile", "128x256", 1, False, False): (19, 527, 271, 544, 144),
    ("tile", "128x256", 1, False, True): (7, 1400, 1400, 544, 144),
    ("tile", "32x64", 1, True, False): (23, 485, 262, 1312, 144), ("tile", "32x64", 1, True, True): (1, 530, 526, 23808, 144),
    ("tile", "64x64", 1, True, False): (15, 758, 502, 1344, 144), ("tile", "64x64", 1, True, True): (2, 538, 538, 13568, 144),
    ("tile", "64x128", 1, True, False): (13, 908, 818, 1312, 144), ("tile", "64x128", 1, True, True): (2, 283, 278, 22336, 144),
    ("tile", "128x128", 1, True, False): (24, 459, 398, 1568, 144),
    ("tile", "128x128", 1, True, True): (2, 292, 251, 26496, 176),
    ("tile", "128x256", 1, True, False): (2, 551, 291, 16480, 1168),
    ("tile", "128x256", 1, True, True): (4, 294, 294, 28128, 1552),
    ("192x192", True): (30, 363, 282, 544, 144), ("192x256", True): (1, 391, 391, 17216, 144),
    ("256x256", False): (15, 739, 554, 672, 144), ("256x256", True): (1, 396, 313, 22016, 208)}


def list_plan(rows, capacity, length):
    plan = pp.pp_pack([length] * rows, capacity)
    assert plan.n_rows == rows
    return plan


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def check(got, v, epi, c0, bf):
    """As check_gemm in test_gpu_quant.py, on the GPU: the sum's conversion and its two products with the scales
    are 3 U of v; SiLU moves a relative error of its argument by at most 1 + |gate|, the exponential's argument
    is rounded twice, and exponential, sum and reciprocal take up to 2 U each."""
    if epi == pp.PP_EPI_RESIDUAL:
        ref = c0 + v
        bound = 3.1 * U * v.abs() + 1.01 * U * ref.abs()
    elif epi == pp.PP_EPI_SWIGLU:
        b = v.unflatten(1, (-1, 2, 16))
        gate, up = b[:, :, 0].flatten(1), b[:, :, 1].flatten(1)
        ref = gate * up / (1 + torch.exp(-gate))
        bound = (6.2 + 6.1 * gate.abs() + 7) * U * ref.abs() + 1e-36
    else:
        ref, bound = v, 3.1 * U * v.abs()
    if bf:
        bound = bound + 2.0 ** -8 * (ref.abs() + bound)
    assert bool(((got - ref).abs() <= bound + 2.0 ** -149).all())


def run(M, N, K, epi, dtype, plan):
    code, t = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(M * 7919 + N * 31 + K)
    a = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8, device="cuda")
    b = torch.randint(-127, 128, (N, K), generator=g, dtype=torch.int8, device="cuda")
    # the products have unit size: codes are uniform, of standard deviation 73
    sa = torch.exp(0.3 * torch.randn(M, generator=g, device="cuda")) / 73
    sb = torch.exp(0.3 * torch.randn(N, generator=g, device="cuda")) / (73 * K ** 0.5)
    cols = N // 2 if epi == pp.PP_EPI_SWIGLU else N
    c0 = torch.randn(M + 1, cols + 8, generator=g, device="cuda").to(t)
    c = c0.clone()
    need = pp.pp_gemm_quant_workspace_size(M, N, K)
    ws = torch.full((need,), 0x5a, dtype=torch.uint8, device="cuda") if need else None
    pp.pp_gemm_quant(code, epi, a, K, sa, b, K, sb, c, cols + 8, M, N, K, ws, None if plan is None else pp.DevicePlan(plan))
    covered = torch.ones(M, dtype=torch.bool, device="cuda")
    if plan is not None:
        covered[:] = False
        for m0 in plan.mtile_m0:
            covered[m0:m0 + 256] = True
    assert torch.equal(c[M], c0[M]) and torch.equal(c[:, cols:], c0[:, cols:])
    assert torch.equal(c[:M][~covered], c0[:M][~covered])
    v = torch.mm(a[covered].double(), b.double().t()).mul_(sa[covered].double()[:, None]).mul_(sb.double())
    check(c[:M, :cols][covered].double(), v, epi, c0[:M, :cols][covered].double(), dtype == "bf16")


EPILOGUES = [(pp.PP_EPI_STORE, "bf16"), (pp.PP_EPI_STORE, "f32"), (pp.PP_EPI_RESIDUAL, "f32"), (pp.PP_EPI_SWIGLU, "bf16"),
             (pp.PP_EPI_SWIGLU, "f32")]


@pytest.mark.parametrize("epi,dtype", EPILOGUES)
@pytest.mark.parametrize("way", ROWS, ids=str)
def test_rows(way, epi, dtype):
    run(*ROWS[way], epi, dtype, None)


@pytest.mark.parametrize("epi,dtype", EPILOGUES)
@pytest.mark.parametrize("way", LISTS, ids=str)
def test_row_tile_list(way, epi, dtype):
    rows, capacity, length, N, K = LISTS[way]
    run(rows * capacity, N, K, epi, dtype, list_plan(rows, capacity, length))


@pytest.mark.parametrize("epi,dtype", [(pp.PP_EPI_STORE, "bf16"), (pp.PP_EPI_SWIGLU, "bf16"), (pp.PP_EPI_RESIDUAL, "f32")])
@pytest.mark.parametrize("M,N,K", [(17, 2 ** 28 - 32, 16), (17, 2 ** 28, 16), (64, 2 ** 28 + 32, 16), (1, 2 ** 30, 16),
                                   (3, 2 ** 31 - 512, 16)])
def test_very_many_columns(M, N, K, epi, dtype):
    """Up to the most columns there may be: the weights repeat, so the columns must.  (Fewer columns are compared
    with float64 above; which kernel takes them does not change a bit.)"""
    code, t = DT[dtype]
    swiglu = epi == pp.PP_EPI_SWIGLU
    period = 4096 + 96
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8, device="cuda")
    b1 = torch.randint(-127, 128, (period, K), generator=g, dtype=torch.int8, device="cuda")
    sa, sb1 = torch.rand(M, generator=g, device="cuda") / 100, torch.rand(period, generator=g, device="cuda") / 100
    times = -(-N // period)
    b, sb = b1.repeat(times, 1), sb1.repeat(times)
    cols, period_c = (N // 2, period // 2) if swiglu else (N, period)
    want = torch.ones((M, period_c), dtype=t, device="cuda")
    pp.pp_gemm_quant(code, epi, a, K, sa, b1, K, sb1, want, period_c, M, period, K)
    c = torch.ones((M, cols), dtype=t, device="cuda")
    need = pp.pp_gemm_quant_workspace_size(M, N, K)
    pp.pp_gemm_quant(code, epi, a, K, sa, b, K, sb, c, cols, M, N, K,
                     torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    whole = cols // period_c
    for m in range(M):
        assert bool((c[m, :whole * period_c].view(whole, period_c) == want[m]).all())
        assert torch.equal(c[m, whole * period_c:], want[m, :cols - whole * period_c])


def test_very_many_rows():
    """The most rows there may be, on as few columns: the rows repeat too."""
    M, N, K, period = 2 ** 31 - 512, 16, 16, 4096 + 96
    g = torch.Generator(device="cuda").manual_seed(9)
    a1 = torch.randint(-127, 128, (period, K), generator=g, dtype=torch.int8, device="cuda")
    b = torch.randint(-127, 128, (N, K), generator=g, dtype=torch.int8, device="cuda")
    sa1, sb = torch.rand(period, generator=g, device="cuda") / 100, torch.rand(N, generator=g, device="cuda") / 100
    want = torch.empty((period, N), dtype=torch.bfloat16, device="cuda")
    pp.pp_gemm_quant(pp.PP_BF16, pp.PP_EPI_STORE, a1, K, sa1, b, K, sb, want, N, period, N, K)
    times = -(-M // period)
    a, sa = a1.repeat(times, 1), sa1.repeat(times)
    c = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    assert pp.pp_gemm_quant_workspace_size(M, N, K) == 0
    pp.pp_gemm_quant(pp.PP_BF16, pp.PP_EPI_STORE, a, K, sa, b, K, sb, c, N, M, N, K)
    whole, step = M // period, 50000
    for i in range(0, whole, step):
        n = min(step, whole - i)
        assert bool((c[i * period:(i + n) * period].view(n, period, N) == want).all())
    assert torch.equal(c[whole * period:], want[:M - whole * period])
