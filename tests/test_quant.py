"""The 8-bit projections' argument checks: every refusal happens on the host, before anything is
enqueued, so nothing here touches a GPU."""
import ctypes

import pytest

from paper_2404_09529_amd import prepack as pp

BF, F32 = pp.PP_BF16, pp.PP_F32
OK, INV, UNS, SMALL = pp.PP_OK, pp.PP_ERR_INVALID_ARG, pp.PP_ERR_UNSUPPORTED, pp.PP_ERR_BUFFER_TOO_SMALL


def _rows(**kw):
    a = dict(dtype=BF, x=0x1000, ldx=256, rows=4, d=256, q=0x2000, ldq=256, scale=0x3004)
    a.update(kw)
    return pp.lib().pp_quantize_rows(a["dtype"], a["x"], a["ldx"], a["rows"], a["d"], a["q"], a["ldq"], a["scale"], None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(dtype=2)), (INV, dict(rows=-1)), (INV, dict(d=0)), (INV, dict(d=-16)), (INV, dict(ldx=240)),
    (INV, dict(ldq=240)), (UNS, dict(d=250)), (UNS, dict(ldx=260)), (UNS, dict(ldq=264)), (INV, dict(x=None)),
    (INV, dict(q=None)), (INV, dict(scale=None)), (UNS, dict(x=0x1008)), (UNS, dict(q=0x2004)),
    (OK, dict(rows=0, x=None, q=None, scale=None))])
def test_quantize_rows_checks(want, kw):
    assert _rows(**kw) == want
    assert (want == OK) == (pp.pp_last_error() == "")
    a = {**dict(dtype=BF, x=0x1000, ldx=256, rows=4, d=256, q=0x2000, ldq=256, scale=0x3004), **kw}
    assert pp.lib().pp_dequantize_rows(a["dtype"], a["q"], a["ldq"], a["scale"], a["rows"], a["d"], a["x"], a["ldx"],
                                       None) == want


def _norm(**kw):
    a = dict(dtype=BF, x=0x1000, add=None, g=0x5000, rows=4, d=256, eps=1e-5, q=0x2000, scale=0x3004)
    a.update(kw)
    return pp.lib().pp_rmsnorm_quant(a["dtype"], a["x"], a["add"], a["g"], a["rows"], a["d"], a["eps"], a["q"],
                                     a["scale"], None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(dtype=-1)), (INV, dict(rows=-1)), (INV, dict(d=0)), (UNS, dict(d=264)), (INV, dict(eps=-1.0)),
    (INV, dict(eps=float("nan"))), (INV, dict(x=None)), (INV, dict(g=None)), (INV, dict(q=None)),
    (INV, dict(scale=None)), (UNS, dict(x=0x1004)), (UNS, dict(add=0x1008)), (UNS, dict(g=0x5008)),
    (UNS, dict(q=0x2008)), (OK, dict(rows=0, x=None))])
def test_rmsnorm_quant_checks(want, kw):
    assert _norm(**kw) == want


def _gemm(**kw):
    a = dict(dtype=BF, epi=pp.PP_EPI_STORE, A=0x1000, lda=256, sa=0x2004, B=0x3000, ldb=256, sb=0x4004, C=0x5000,
             ldc=512, M=4096, N=512, K=256, plan=None, ws=0x10000, bytes=1 << 40)
    a.update(kw)
    return pp.lib().pp_gemm_quant(a["dtype"], a["epi"], a["A"], a["lda"], a["sa"], a["B"], a["ldb"], a["sb"], a["C"],
                                  a["ldc"], a["M"], a["N"], a["K"], a["plan"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(dtype=9)), (INV, dict(epi=3)), (INV, dict(epi=-1)), (INV, dict(M=-1)), (INV, dict(N=0)),
    (INV, dict(K=0)), (INV, dict(lda=240)), (INV, dict(ldb=240)), (INV, dict(ldc=496)),
    (UNS, dict(K=248)), (UNS, dict(N=504)), (UNS, dict(N=496, epi=pp.PP_EPI_SWIGLU, ldc=256)),
    (UNS, dict(K=131072, lda=131072, ldb=131072)), (UNS, dict(lda=264)), (UNS, dict(ldb=264)), (UNS, dict(ldc=514)),
    (UNS, dict(M=2 ** 31 - 511)), (UNS, dict(N=2 ** 31 - 496, ldc=2 ** 31)), (UNS, dict(lda=8388608)), (UNS, dict(ldb=8388608)), (INV, dict(A=None)), (INV, dict(sa=None)),
    (INV, dict(B=None)), (INV, dict(sb=None)), (INV, dict(C=None)), (UNS, dict(A=0x1008)), (UNS, dict(B=0x3004)),
    (UNS, dict(C=0x5008)), (OK, dict(M=0, A=None, B=None, C=None, ws=None, bytes=0))])
def test_gemm_quant_checks(want, kw):
    assert _gemm(**kw) == want


def test_gemm_quant_plan_checks():
    arrays = {n: 0x1000 for n in ("seg_prompt", "seg_start", "seg_len", "prompt_kv_off", "slot_seg", "slot_pos",
                                  "slot_kv", "qtile_seg", "qtile_q0", "mtile_m0")}

    def plan(**kw):
        return ctypes.byref(pp.PPDPlan(**{**dict(k=2, capacity=256, n_rows=2, max_len=200, total_len=300, n_qtiles=3,
                                                 n_mtiles=2, **arrays), **kw}))

    assert _gemm(plan=plan(), M=513) == INV                     # M is not the plan's slots
    assert _gemm(plan=plan(mtile_m0=0), M=512) == INV
    assert _gemm(plan=plan(n_mtiles=3), M=512) == INV
    empty = plan(k=0, capacity=0, n_rows=0, max_len=0, total_len=0, n_qtiles=0, n_mtiles=0)
    assert _gemm(plan=empty, M=0) == OK


def test_gemm_quant_workspace():
    with pytest.raises(pp.PrepackError):
        pp.pp_gemm_quant_workspace_size(-1, 512, 256)
    with pytest.raises(pp.PrepackError):
        pp.pp_gemm_quant_workspace_size(1, 0, 256)
    assert pp.pp_gemm_quant_workspace_size(0, 512, 256) == 0
    for M, N, K in [(1, 4096, 4096), (48, 4096, 14336), (200, 2048, 5504), (27721, 22016, 4096)]:
        need = pp.pp_gemm_quant_workspace_size(M, N, K)
        assert 0 <= need <= 16 * M * N * 4 + 4096
        if need:
            kw = dict(M=M, N=N, K=K, lda=K, ldb=K, ldc=N)
            assert _gemm(ws=None, **kw) == INV
            assert _gemm(ws=0x10010, **kw) == INV
            assert _gemm(bytes=need - 1, **kw) == SMALL
