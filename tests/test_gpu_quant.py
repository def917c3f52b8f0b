"""8-bit projections on the GPU, through the C ABI, against float64.

Integer sums are exact, so every bound below counts roundings: 2^-24 of the value for a float32
operation, 2^-8 for storing bf16."""
import numpy as np
import pytest
import torch

from oracle import decoder as D
from paper_2404_09529_amd import prepack as pp

from .gpu_util import require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": (pp.PP_BF16, torch.bfloat16), "f32": (pp.PP_F32, torch.float32)}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def h64(t):
    return t.double().cpu().numpy()


# ----------------------------------------------------------------------------- rows in 8 bits
def check_codes(y, q, scale, rel):
    """q, scale against the float64 rows y, which the kernel saw with relative error rel.
    scale = max * (1 / 127) with a rounding in each.  What is rounded to an integer is y / scale, of at most 127
    and off by 2 rel (once in y, once in the scale) and two more roundings; a code by half a step
    more.  (scale is the one the kernel wrote.)"""
    top = np.abs(y).max(axis=1)
    assert np.all(np.abs(scale - top / 127) <= (rel + 2.01 * U) * top / 127 + 2.0 ** -149)
    assert np.abs(q).max(initial=0) <= 127
    live = scale > 0
    assert np.all(q[~live] == 0)
    t = y[live] / scale[live][:, None]
    assert np.all(np.abs(q[live] - t) <= 0.5 + 127.1 * (2 * U + 2 * rel))


ROWS = [(1, 16), (1, 4096), (3, 48), (5, 688), (65, 1024), (7, 1040), (130, 2064), (33, 5120), (9, 8192), (4, 14336),
        (3, 20000), (2, 33040), (2, 70000), (3, 140000), (4100, 256), (2500, 688)]


@pytest.mark.parametrize("rows,d", ROWS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_rows(rows, d, dtype):
    code, t = DT[dtype]
    g = torch.Generator().manual_seed(rows * 100000 + d)
    x = (torch.randn(rows, d + 32, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))).to(t).cuda()
    q = torch.full((rows + 1, d + 16), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((rows + 1,), -3.0, device="cuda")
    pp.pp_quantize_rows(code, x, d + 32, rows, d, q, d + 16, scale)
    y, s = h64(x[:, :d]), h64(scale)
    check_codes(y, h64(q)[:rows, :d], s[:rows], 0.0)
    assert np.array_equal(s[:rows], (np.abs(y).max(1).astype(np.float32) * (np.float32(1) / np.float32(127))).astype(np.float64))
    with np.errstate(invalid="ignore"):                        # the float32 quotient, ties to even
        want = np.rint(y.astype(np.float32) / s[:rows, None].astype(np.float32))
    assert np.array_equal(h64(q)[:rows, :d], want)
    assert bool((q[rows] == 55).all()) and bool((q[:, d:] == 55).all()) and s[rows] == -3.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 2048, 20000, 140000])
def test_quantize_rows_special(dtype, d):
    """Zero rows, magnitudes at both ends of the type, ties, and rows with NaN or infinities."""
    code, t = DT[dtype]
    x = torch.zeros(12, d)
    x[1, 5] = 3e38
    x[1, 6] = -3e38
    x[2, 0] = 1e-40                                            # a denormal alone
    x[3] = torch.linspace(-1.2e-38, 1.2e-38, d)
    x[4, :] = 127.0 * 2.0 ** -130                              # the scale itself is denormal
    x[4, 1::2] = -2.0 ** -130
    x[5, :4] = torch.tensor([127.0, 0.5, 1.5, -2.5])           # ties go to the even code
    x[6, d - 1] = float("nan")
    x[7, 0] = float("inf")
    x[8, 3] = -float("inf")
    x[9] = -0.0
    x[10] = 1e-45                                              # scale rounds to 0
    x[11] = torch.randn(d, generator=torch.Generator().manual_seed(1))
    x = x.to(t).cuda()
    q = torch.full((12, d), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((12,), -3.0, device="cuda")
    pp.pp_quantize_rows(code, x, d, 12, d, q, d, scale)
    y, k, s = h64(x), h64(q), h64(scale)
    bad = [6, 7, 8]
    assert np.isnan(s[bad]).all() and (k[bad] == 0).all()
    good = [i for i in range(12) if i not in bad]
    want = (np.abs(y[good]).max(1).astype(np.float32) * (np.float32(1) / np.float32(127))).astype(np.float64)
    assert np.array_equal(s[good], want)
    for i in good:
        if s[i] == 0:
            assert (k[i] == 0).all()
        else:
            assert np.all(np.abs(k[i] - np.clip(y[i] / s[i], -127, 127)) <= 0.5 + 127.1 * 2 * U)
    assert k[5, :4].tolist() == [127, 0, 2, -2]


@pytest.mark.parametrize("rows,d", ROWS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dequantize_rows(rows, d, dtype):
    """One float32 product, rounded once more to bf16: equal to the same in numpy and torch."""
    code, t = DT[dtype]
    g = torch.Generator().manual_seed(rows * 100000 + d + 2)
    q = torch.randint(-128, 128, (rows, d + 48), generator=g, dtype=torch.int8)
    scale = torch.exp(20 * torch.randn(rows, generator=g))
    scale[-1] = float("nan")
    if rows > 2:
        scale[0], scale[1] = 0.0, 1e-45
    x0 = torch.full((rows + 1, d + 16), 9.0).to(t)
    x = x0.cuda()
    pp.pp_dequantize_rows(code, q.cuda(), d + 48, scale.cuda(), rows, d, x, d + 16)
    got = x.cpu()
    want = (q[:, :d].float() * scale[:, None]).to(t)
    assert torch.equal(got[:rows - 1, :d], want[:-1]) and bool(got[rows - 1, :d].isnan().all())
    assert torch.equal(got[rows], x0[rows]) and torch.equal(got[:, d:], x0[:, d:])


def rel_norm(d):
    """Relative error of RMSNorm in float32: a lane adds at most d / 64 squares in turn, and up to ten
    partial sums follow (half of it after the square root); division, eps, root, two products."""
    return (d / 128 + 5 + 6) * U


@pytest.mark.parametrize("rows,d", ROWS)
@pytest.mark.parametrize("add", [None, "bf16", "f32"])
def test_rmsnorm_quant(rows, d, add):
    code, t = DT[add or "bf16"]
    g = torch.Generator().manual_seed(rows * 100000 + d + 1)
    x = torch.randn(rows + 1, d, generator=g) * torch.exp(torch.randn(rows + 1, 1, generator=g))
    gain = 1 + 0.3 * torch.randn(d, generator=g)
    a = None if add is None else (0.5 * torch.randn(rows, d, generator=g)).to(t)
    xd, q, scale = x.cuda(), torch.full((rows + 1, d), 55, dtype=torch.int8, device="cuda"), torch.full((rows + 1,), -3.0, device="cuda")
    pp.pp_rmsnorm_quant(code, xd, None if a is None else a.cuda(), gain.cuda(), rows, d, 1e-5, q, scale)
    want = x.clone()
    if a is not None:
        want[:rows] += a.float()
    assert torch.equal(xd.cpu(), want)                         # the sum is one float32 addition
    y = want[:rows].double().numpy()
    y = y / np.sqrt((y * y).mean(axis=1, keepdims=True) + 1e-5) * gain.double().numpy()
    check_codes(y, h64(q)[:rows], h64(scale)[:rows], rel_norm(d))
    assert bool((q[rows] == 55).all()) and float(scale[rows]) == -3.0


@pytest.mark.parametrize("d", [64, 4096, 20000])
def test_rmsnorm_quant_special(d):
    """A zero row, rows with NaN or an infinity (also brought in by add), eps that dominates."""
    x = torch.randn(6, d, generator=torch.Generator().manual_seed(2))
    a = torch.zeros(6, d)
    x[0] = 0
    x[1, 7] = float("nan")
    a[2, d - 2] = float("inf")
    x[3] *= 1e-30                                              # mean of squares underflows to eps alone
    x[4, 0], a[4, 0] = 3e38, 3e38                              # overflows in the sum
    xd, q, scale = x.cuda(), torch.full((6, d), 55, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    pp.pp_rmsnorm_quant(pp.PP_F32, xd, a.cuda(), torch.ones(d, device="cuda"), 6, d, 1e-5, q, scale)
    k, s = h64(q), h64(scale)
    assert s[0] == 0 and (k[0] == 0).all()
    for i in (1, 2, 4):
        assert np.isnan(s[i]) and (k[i] == 0).all()
    for i in (3, 5):
        y = x[i:i + 1].double().numpy()
        y = y / np.sqrt((y * y).mean() + 1e-5)
        check_codes(y, k[i:i + 1], s[i:i + 1], rel_norm(d))


# ----------------------------------------------------------------------------- GEMM
def codes(g, *shape):
    return torch.randint(-127, 128, shape, generator=g, dtype=torch.int8)


def product(a, sa, b, sb):
    """(A B^T) scaled, in float64 (the integer sums stay below 2^53, so they are exact in any order)."""
    a, sa, b, sb = (t.cuda().double() for t in (a, sa, b, sb))
    return torch.mm(a, b.t()).mul_(sa[:, None]).mul_(sb).cpu().numpy()


def swiglu(v):
    v = v.reshape(v.shape[0], -1, 2, 16)
    g, u = v[:, :, 0].reshape(v.shape[0], -1), v[:, :, 1].reshape(v.shape[0], -1)
    return g, u, D.silu(g) * u


def check_gemm(got, v, epi, c0, bf):
    """The sum's conversion and its two products with the scales: 3 U of v.  SiLU moves a relative
    error of its argument by at most 1 + |gate|; its exponential's argument is rounded twice (|gate| U each,
    with log2 e a little more) and exponential, sum and reciprocal take up to 2 U each."""
    if epi == pp.PP_EPI_RESIDUAL:
        ref = c0 + v
        bound = 3.1 * U * np.abs(v) + 1.01 * U * np.abs(ref)
    elif epi == pp.PP_EPI_SWIGLU:
        g, _, ref = swiglu(v)
        bound = ((3.1 + 3.1) + 3.1 * np.abs(g) + 3 * np.abs(g) + 7) * U * np.abs(ref) + 1e-36
    else:
        ref, bound = v, 3.1 * U * np.abs(v)
    if bf:
        bound = bound + 2.0 ** -8 * (np.abs(ref) + bound)
    assert np.all(np.abs(got - ref) <= bound + 2.0 ** -149)


SIZES = [(1, 32, 16), (1, 512, 64), (2, 96, 144), (3, 32, 4096), (7, 4096, 688), (16, 256, 4112), (17, 544, 1024),
         (31, 2048, 5504), (32, 6144, 512), (33, 160, 1040), (48, 1024, 4096), (64, 4096, 2048), (65, 512, 272),
         (100, 2080, 11008), (128, 128, 128), (129, 2048, 1360), (255, 608, 4096), (256, 4096, 64), (344, 2048, 5504),
         (513, 1056, 2000), (700, 11008, 512), (1309, 2048, 1376), (2926, 6144, 144), (4097, 800, 256),
         # the other ways a call may go: two and four column blocks of the few-row kernel and more than a round
         # of them, tiles of 64 x 128 and 128 x 256, 192 x 192 (700 rows above), 192 x 256 and 256 x 256, whole
         # rounds of 256-row tiles with smaller ones after them
         (2800, 1600, 656), (640, 12800, 400), (2500, 2080, 1040), (12, 8192, 1040), (14, 12288, 528), (9, 20000, 144), (3000, 4096, 1040), (3500, 4064, 1040), (5000, 4064, 1040),
         (8500, 4096, 1040), (33000, 544, 144),
         # and two column blocks for 64 rows, 64 x 128 tiles alone, shares of K of the smaller tiles, 32 x 64 and
         # 64 x 64 tiles after whole rounds
         (39, 4160, 80), (257, 3808, 64), (41, 32, 4544), (41, 2784, 6448), (65, 5888, 6464), (38, 32, 5392),
         (90, 2240, 12496), (66, 6016, 7824), (520, 23840, 128),
         (6235, 2656, 240)]


def gemm_case(M, N, K, seed=0):
    g = torch.Generator().manual_seed(M * 7919 + N * 31 + K + seed)
    a, b = codes(g, M, K), codes(g, N, K)
    # the products have unit size: codes are uniform, of standard deviation 73
    sa = torch.exp(0.3 * torch.randn(M, generator=g)) / 73
    sb = torch.exp(0.3 * torch.randn(N, generator=g)) / (73 * K ** 0.5)
    return g, a, sa, b, sb


def gpu_gemm(epi, code, a, sa, b, sb, c, M, N, K, lda=None, ldb=None, ldc=None, dplan=None):
    need = pp.pp_gemm_quant_workspace_size(M, N, K)
    ws = torch.full((max(need, 1),), 0x5a, dtype=torch.uint8, device="cuda")
    pp.pp_gemm_quant(code, epi, a, lda or K, sa, b, ldb or K, sb, c, ldc or c.shape[1], M, N, K, ws, dplan)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("epi,dtype", [(pp.PP_EPI_STORE, "bf16"), (pp.PP_EPI_STORE, "f32"), (pp.PP_EPI_RESIDUAL, "f32"),
                                       (pp.PP_EPI_SWIGLU, "bf16"), (pp.PP_EPI_SWIGLU, "f32")])
def test_gemm_quant(M, N, K, epi, dtype):
    """Strided operands and output; columns past the output's and the row past M are left alone."""
    code, t = DT[dtype]
    g, a, sa, b, sb = gemm_case(M, N, K)
    cols = N // 2 if epi == pp.PP_EPI_SWIGLU else N
    A = torch.nn.functional.pad(a, (0, 48), value=99).cuda()
    B = torch.nn.functional.pad(b, (0, 16), value=-77).cuda()
    c0 = torch.randn(M + 1, cols + 12, generator=g).to(t)
    c = c0.cuda()
    gpu_gemm(epi, code, A, sa.cuda(), B, sb.cuda(), c, M, N, K, K + 48, K + 16, cols + 12)
    got = c.cpu()
    assert torch.equal(got[M], c0[M]) and torch.equal(got[:, cols:], c0[:, cols:])
    check_gemm(h64(got[:M, :cols]), product(a, sa, b, sb), epi, h64(c0[:M, :cols]), dtype == "bf16")


@pytest.mark.parametrize("M,N,K", [(1, 2048, 5504), (20, 4096, 4096), (65, 2048, 5504), (300, 6144, 1040), (1309, 2048, 688)])
@pytest.mark.parametrize("epi", [pp.PP_EPI_STORE, pp.PP_EPI_RESIDUAL, pp.PP_EPI_SWIGLU])
def test_gemm_quant_rows_do_not_depend_on_the_batch(M, N, K, epi):
    big = 4096 + M
    g, a, sa, b, sb = gemm_case(big, N, K)
    cols = N // 2 if epi == pp.PP_EPI_SWIGLU else N
    t = torch.float32 if epi == pp.PP_EPI_RESIDUAL else torch.bfloat16
    c0 = torch.randn(big, cols, generator=g).to(t).cuda()
    small, large = c0[:M].clone(), c0.clone()
    a, sa, b, sb = a.cuda(), sa.cuda(), b.cuda(), sb.cuda()
    gpu_gemm(epi, pp.PP_BF16, a, sa, b, sb, small, M, N, K)
    gpu_gemm(epi, pp.PP_BF16, a, sa, b, sb, large, big, N, K)
    assert torch.equal(small, large[:M])


@pytest.mark.parametrize("M", [1, 40, 300])
def test_gemm_quant_extremes(M):
    """The largest sums 32 bits hold (codes of -128 over the longest K), and scales that are zero, NaN or
    large enough to overflow."""
    N, K = 64, 131056
    a = torch.full((M, K), -128, dtype=torch.int8)
    b = torch.full((N, K), -128, dtype=torch.int8)
    b[1] = 127
    sa, sb = torch.ones(M), torch.ones(N)
    sb[2], sb[3], sb[4] = 0.0, float("nan"), 1e38
    sa[M - 1] = 0.5 if M > 1 else 1.0
    c = torch.empty(M, N, device="cuda")
    gpu_gemm(pp.PP_EPI_STORE, pp.PP_F32, a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), c, M, N, K)
    got = h64(c)
    assert np.all(got[:, 0] == K * 16384 * sa.double().numpy())
    assert np.all(got[:, 1] == float(np.float32(-K * 128 * 127)) * sa.double().numpy())
    assert np.all(got[:, 2] == 0) and np.isnan(got[:, 3]).all() and np.all(got[:, 4] == np.inf)


@pytest.mark.parametrize("epi", [pp.PP_EPI_STORE, pp.PP_EPI_RESIDUAL, pp.PP_EPI_SWIGLU])
@pytest.mark.parametrize("lengths,N,K", [([700, 700, 700, 600, 600, 600, 300], 4096, 2048),
                                         ([700, 700, 700, 600, 600, 600, 300], 544, 208),
                                         ([700] * 18, 1024, 2064), ([700] * 18, 1280, 2064)])
def test_gemm_quant_plan_row_tiles(epi, lengths, N, K):
    """With a plan exactly its row tiles are computed; tiles of padding alone keep what they held."""
    plan = pp.pp_pack(lengths, 1024)
    T = plan.n_slots
    assert plan.n_mtiles < T // 256
    g, a, sa, b, sb = gemm_case(T, N, K)
    cols = N // 2 if epi == pp.PP_EPI_SWIGLU else N
    t = torch.float32 if epi == pp.PP_EPI_RESIDUAL else torch.bfloat16
    c0 = torch.randn(T, cols, generator=g).to(t)
    c = c0.cuda()
    gpu_gemm(epi, pp.PP_BF16, a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), c, T, N, K, dplan=pp.DevicePlan(plan))
    covered = torch.zeros(T, dtype=torch.bool)
    for m0 in plan.mtile_m0:
        covered[m0:m0 + 256] = True
    got = c.cpu()
    assert torch.equal(got[~covered], c0[~covered])
    check_gemm(h64(got[covered]), product(a[covered], sa[covered], b, sb), epi, h64(c0[covered]), t == torch.bfloat16)


@pytest.mark.parametrize("M,N,K", [(66000, 33024, 128), (66000, 256, 33024), (256, 66016, 33024), (20, 66016, 33024)])
def test_gemm_quant_offsets_past_32_bits(M, N, K):
    """Operands and outputs of more than 2^31 elements: rows and columns at both ends."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8, device="cuda")
    b = torch.randint(-127, 128, (N, K), generator=g, dtype=torch.int8, device="cuda")
    sa, sb = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda") / K
    c = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    gpu_gemm(pp.PP_EPI_STORE, pp.PP_BF16, a, sa, b, sb, c, M, N, K)
    m = torch.tensor([0, 1, M // 2, M - 2, M - 1], device="cuda")
    n = torch.cat([torch.arange(0, 40), torch.arange(N // 2, N // 2 + 24), torch.arange(N - 40, N)]).cuda()
    check_gemm(h64(c[m][:, n]), product(a[m].cpu(), sa[m].cpu(), b[n].cpu(), sb[n].cpu()), pp.PP_EPI_STORE, None, True)


def test_rows_offsets_past_32_bits():
    rows, d = 140000, 16384
    x = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda")
    x.zero_()
    ends = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    x[ends] = torch.randn((5, d), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").bfloat16()
    q, scale = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    pp.pp_quantize_rows(pp.PP_BF16, x, d, rows, d, q, d, scale)
    check_codes(h64(x[ends]), h64(q[ends]), h64(scale[ends]), 0.0)
    x2 = torch.empty_like(x)
    pp.pp_dequantize_rows(pp.PP_BF16, q, d, scale, rows, d, x2, d)
    assert torch.equal(x2[ends], (q[ends].float() * scale[ends][:, None]).bfloat16())
    assert int((scale != 0).sum()) == 5


def test_rows_more_than_a_launch_dimension_holds():
    """17 million rows of 16 values: more than 2^32 threads in one dimension, were each row a workgroup."""
    rows, d = 17_000_003, 16
    x = (torch.arange(rows, device="cuda") % 1000).float()[:, None].repeat(1, d)
    q, scale = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    pp.pp_quantize_rows(pp.PP_F32, x, d, rows, d, q, d, scale)
    assert torch.equal(scale, x[:, 0] * (torch.ones((), device="cuda") / 127))
    assert torch.equal(q, ((x > 0) * 127).to(torch.int8))
    pp.pp_rmsnorm_quant(pp.PP_F32, x, None, torch.ones(d, device="cuda"), rows, d, 0.5, q, scale)
    assert torch.equal(q, ((x > 0) * 127).to(torch.int8))


def test_rows_of_nearly_2_31_values():
    """The longest row: three values that are not 0, at its ends and in the middle."""
    d = 2 ** 31 - 16
    at = torch.tensor([0, d // 2 + 1, d - 1], device="cuda")
    val = torch.tensor([-1.0, 2.0, 3.0], device="cuda")
    want = torch.tensor([-42, 85, 127], dtype=torch.int8, device="cuda")       # 127 / 3, 254 / 3, 127
    q, scale = torch.empty(d, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    for t, code in ((torch.bfloat16, pp.PP_BF16), (torch.float32, pp.PP_F32)):
        x = torch.zeros(d, dtype=t, device="cuda")
        x[at] = val.to(t)
        q.fill_(9)
        pp.pp_quantize_rows(code, x, d, 1, d, q, d, scale)
        assert torch.equal(q[at], want) and int(q.count_nonzero()) == 3
        pp.pp_dequantize_rows(code, q, d, scale, 1, d, x, d)
        assert torch.equal(x[at], (want.float() * scale).to(t)) and int(x.count_nonzero()) == 3
    q.fill_(9)
    pp.pp_rmsnorm_quant(pp.PP_F32, x, None, torch.ones(d, device="cuda"), 1, d, 0.0, q, scale)
    assert torch.equal(q[at], want) and int(q.count_nonzero()) == 3


@pytest.mark.parametrize("M,N,K", [(7, 512, 272), (100, 512, 272), (1309, 2048, 688)])
def test_gemm_quant_scales_at_any_float(M, N, K):
    g, a, sa, b, sb = gemm_case(M, N, K, 5)
    sa1, sb1 = torch.cat([torch.zeros(1), sa]).cuda()[1:], torch.cat([torch.zeros(3), sb]).cuda()[3:]
    c = torch.empty(M, N, device="cuda")
    gpu_gemm(pp.PP_EPI_STORE, pp.PP_F32, a.cuda(), sa1, b.cuda(), sb1, c, M, N, K)
    check_gemm(h64(c), product(a, sa, b, sb), pp.PP_EPI_STORE, None, False)


def test_gemm_quant_on_two_streams_at_once():
    """Calls that split K (a workspace each) and calls that do not, on two streams, each on its own buffers."""
    M, N, K = 64, 4096, 14336
    assert pp.pp_gemm_quant_workspace_size(M, N, K) > 0
    g, a, sa, b, sb = gemm_case(M, N, K, 6)
    a, sa, b, sb = a.cuda(), sa.cuda(), b.cuda(), sb.cuda()
    want = torch.empty(M, N, device="cuda")
    gpu_gemm(pp.PP_EPI_STORE, pp.PP_F32, a, sa, b, sb, want, M, N, K)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(pp.pp_gemm_quant_workspace_size(M, N, K), dtype=torch.uint8, device="cuda") for _ in streams]
    out = [[torch.empty(M, N, device="cuda") for _ in range(10)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(10):
        for s, w, o in zip(streams, ws, out):
            pp.pp_gemm_quant(pp.PP_F32, pp.PP_EPI_STORE, a, K, sa, b, K, sb, o[i], N, M, N, K, w, None, s)
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for o in out for t in o)


# ----------------------------------------------------------------------------- together
class Layer:
    """One decoder layer in 8 bits over a packed batch, as a caller assembles it from the single steps."""

    def __init__(self, lengths, capacity, seed, H=4, Hkv=2, d=512, F=1024):
        g = torch.Generator().manual_seed(seed)
        self.plan = pp.pp_pack(lengths, capacity)
        self.dplan = pp.DevicePlan(self.plan)
        self.H, self.Hkv, self.d, self.F, hd, kvw = H, Hkv, d, F, H * 128, Hkv * 128
        self.cfg = pp.PPConfig(n_layers=1, d_model=d, n_heads=H, n_kv_heads=Hkv, head_dim=128, ffn_dim=F, vocab=100,
                               dtype=pp.PP_BF16, rms_eps=1e-5, rope_theta=1e4)
        T = self.T = self.plan.n_slots
        self.gains = [(1 + 0.1 * torch.randn(d, generator=g)).cuda() for _ in range(2)]
        w = [torch.randn(n, k, generator=g) / k ** 0.5 for n, k in
             [(hd + 2 * kvw, d), (d, hd), (F, d), (F, d), (d, F)]]
        w[2:4] = [pp.interleave_gate_up(w[2], w[3])]
        self.w = []
        for x in w:                                            # wqkv, wo, w_gateup, w_down in 8 bits
            n, k = x.shape
            q, s = torch.empty((n, k), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
            pp.pp_quantize_rows(pp.PP_F32, x.cuda(), k, n, k, q, k, s)
            self.w.append((q, s))
        def buf(*shape, dtype=torch.bfloat16):
            return torch.zeros(shape, dtype=dtype, device="cuda")
        self.x0 = torch.randn(T, d, generator=g).cuda()
        self.x0[torch.from_numpy(self.plan.slot_seg < 0).cuda()] = 0
        self.x = self.x0.clone()
        self.qkv, self.attn, self.o, self.act = buf(T, hd + 2 * kvw), buf(T, hd), buf(T, d), buf(T, F)
        self.kc, self.vc = buf(self.plan.total_len, kvw), buf(self.plan.total_len, kvw)
        self.table = buf(self.plan.max_len * 64 * 2, dtype=torch.float32)
        widths = [d, hd, d, F]
        self.q = [buf(T, k, dtype=torch.int8) for k in widths]
        self.s = [buf(T, dtype=torch.float32) for _ in widths]
        self.ws = torch.empty(max(1, max(pp.pp_gemm_quant_workspace_size(T, q.shape[0], q.shape[1]) for q, _ in self.w)),
                              dtype=torch.uint8, device="cuda")

    def gemm(self, i, epi, c):
        (wq, wsc), q = self.w[i], self.q[i]
        n, k = wq.shape
        pp.pp_gemm_quant(pp.PP_BF16, epi, q, k, self.s[i], wq, k, wsc, c, c.shape[1], self.T, n, k, self.ws, self.dplan)

    def rows(self, i, x):
        d = x.shape[1]
        pp.pp_quantize_rows(pp.PP_BF16, x, d, self.T, d, self.q[i], d, self.s[i])

    def __call__(self):
        cfg, dp, T = self.cfg, self.dplan, self.T
        pp.pp_rmsnorm_quant(pp.PP_BF16, self.x, None, self.gains[0], T, self.d, 1e-5, self.q[0], self.s[0])
        self.gemm(0, pp.PP_EPI_STORE, self.qkv)
        pp.pp_rope(cfg, dp, self.qkv, self.table)
        pp.pp_kv_scatter(cfg, dp, self.qkv, self.kc, self.vc)
        pp.pp_attention(cfg, dp, self.qkv, self.qkv.shape[1], self.kc, self.vc, self.attn)
        self.rows(1, self.attn)
        self.gemm(1, pp.PP_EPI_STORE, self.o)
        pp.pp_rmsnorm_quant(pp.PP_BF16, self.x, self.o, self.gains[1], T, self.d, 1e-5, self.q[2], self.s[2])
        self.gemm(2, pp.PP_EPI_SWIGLU, self.act)
        self.rows(3, self.act)
        self.gemm(3, pp.PP_EPI_RESIDUAL, self.x)


@pytest.mark.parametrize("lengths,capacity", [([3, 150, 40, 1, 77], 256), ([300, 200, 513, 64, 20, 20], 600), ([1], 1)])
def test_layer_in_8_bits(lengths, capacity):
    """Every step against float64 on the values that the step before left."""
    L = Layer(lengths, capacity, seed=sum(lengths))
    d, T = L.d, L.T
    real = L.plan.slot_seg >= 0
    mask = torch.from_numpy(real)
    L()
    q = [h64(t)[real] for t in L.q]
    s = [h64(t)[real] for t in L.s]
    w = [(t.cpu(), sc.cpu()) for t, sc in L.w]
    rows = lambda i: (L.q[i].cpu()[mask], L.s[i].cpu()[mask], *w[i])

    def norm(x, gain):
        return x / np.sqrt((x * x).mean(axis=1, keepdims=True) + 1e-5) * h64(gain)

    x0 = h64(L.x0)[real]
    check_codes(norm(x0, L.gains[0]), q[0], s[0], rel_norm(d))
    # queries, keys and values after RoPE: one bf16 rounding before it and one after, on pairs
    qkv = product(*rows(0))
    pos = L.plan.slot_pos[real]
    ang = pos[:, None] * 1e4 ** (-np.arange(64) / 64)
    c, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
    heads = qkv.reshape(len(qkv), -1, 128)
    n_rot = L.H + L.Hkv
    lo, hi = heads[:, :n_rot, :64], heads[:, :n_rot, 64:]
    rot = np.concatenate([np.concatenate([lo * c - hi * sn, hi * c + lo * sn], axis=2), heads[:, n_rot:]], axis=1)
    size = np.sqrt(np.square(lo) + np.square(hi))
    size = np.concatenate([np.concatenate([size, size], axis=2), np.abs(heads[:, n_rot:])], axis=1)
    got = h64(L.qkv)[real].reshape(heads.shape)
    assert np.all(np.abs(got - rot) <= 2.5 * 2.0 ** -8 * size + 1e-6)   # sqrt(2) 2^-8 before, 2^-8 after
    check_codes(h64(L.attn)[real], q[1], s[1], 0.0)
    o = product(*rows(1))
    check_gemm(h64(L.o)[real], o, pp.PP_EPI_STORE, None, True)
    x1 = (L.x0.cpu() + L.o.cpu().float())[mask].double().numpy()
    check_codes(norm(x1, L.gains[1]), q[2], s[2], rel_norm(d))
    check_gemm(h64(L.act)[real], product(*rows(2)), pp.PP_EPI_SWIGLU, None, True)
    check_codes(h64(L.act)[real], q[3], s[3], 0.0)
    check_gemm(h64(L.x)[real], product(*rows(3)), pp.PP_EPI_RESIDUAL, x1, False)


def test_layer_in_8_bits_captured_and_on_another_stream():
    """The same bits from a side stream and from a graph, replayed with eager work in between."""
    L = Layer([3, 150, 40, 1, 77], 256, seed=5)
    L()
    want = L.x.clone()
    side = torch.cuda.Stream()
    L.x.copy_(L.x0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(L.x, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.x.copy_(L.x0)
        L()
    for _ in range(3):
        L.x.fill_(7)
        L.ws.fill_(0x5a)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(L.x, want)
        L.x.copy_(L.x0)
        L()
        assert torch.equal(L.x, want)
