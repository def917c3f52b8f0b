"""The paged cache and sampling on the CPU: every refusal happens on the host before anything is enqueued, and
the index arithmetic of the kernels (``csrc/paged.h``) is asked through ``tests/host/paged_index.cpp``."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from paper_2404_09529_amd import prepack as pp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, F32 = pp.PP_BF16, pp.PP_F32
OK, INV, UNS, SMALL = pp.PP_OK, pp.PP_ERR_INVALID_ARG, pp.PP_ERR_UNSUPPORTED, pp.PP_ERR_BUFFER_TOO_SMALL


def _cfg(**kw):
    return pp.PPConfig(**{**dict(n_layers=1, d_model=512, n_heads=4, n_kv_heads=2, head_dim=128, ffn_dim=1024, vocab=1000,
                                 dtype=BF, rms_eps=1e-5, rope_theta=1e4), **kw})


def _cache(**kw):
    return pp.PPPagedCache(**{**dict(kv_type=pp.PP_KV_BF16, k=3, page_size=16, max_pages=4, n_pages=9, page_table=0x1004,
                                     k_pages=0x2000, v_pages=0x3000, k_scale=None, v_scale=None), **kw})


# what is wrong with the cache or the config: every entry point says the same
CACHES = [
    (INV, {}, dict(kv_type=3)), (INV, {}, dict(kv_type=-1)), (INV, {}, dict(k=-1)), (INV, {}, dict(max_pages=-1)),
    (INV, {}, dict(n_pages=0)), (INV, {}, dict(page_size=0)), (INV, {}, dict(page_size=-16)),
    (UNS, {}, dict(page_size=24)), (UNS, {}, dict(kv_type=pp.PP_KV_F32)),
    (UNS, dict(dtype=F32), {}), (UNS, {}, dict(n_pages=1 << 27)), (UNS, {}, dict(k=1 << 21)),
    (UNS, dict(head_dim=64), {}), (UNS, dict(n_heads=3), {}), (INV, dict(n_layers=0), {}), (INV, dict(dtype=2), {})]
BUFFERS = [
    (INV, {}, dict(page_table=None)), (INV, {}, dict(k_pages=None)), (INV, {}, dict(v_pages=None)),
    (UNS, {}, dict(k_pages=0x2008)), (UNS, {}, dict(v_pages=0x3004)),
    (INV, {}, dict(kv_type=pp.PP_KV_I8, k_scale=0x4000)), (INV, {}, dict(kv_type=pp.PP_KV_I8, v_scale=0x4000))]
NOTHING = dict(k=0, page_table=None, k_pages=None, v_pages=None)


def _rows(cfg=None, cache=None, **kw):
    a = {**dict(seq=0x5004, pos=0x5104, rows=7, k=0x6000, ldk=256, v=0x7000, ldv=256), **kw}
    got = [f(ctypes.byref(_cfg(**(cfg or {}))), ctypes.byref(_cache(**(cache or {}))), a["seq"], a["pos"], a["rows"], a["k"],
             a["ldk"], a["v"], a["ldv"], None) for f in (pp.lib().pp_paged_write, pp.lib().pp_paged_read)]
    assert got[0] == got[1] and (got[0] == OK) == (pp.pp_last_error() == "")
    return got[0]


@pytest.mark.parametrize("want,cfg,cache", CACHES + BUFFERS)
def test_rows_cache(want, cfg, cache):
    assert _rows(cfg, cache) == want


@pytest.mark.parametrize("want,kw", [
    (INV, dict(rows=-1)), (INV, dict(ldk=248)), (INV, dict(ldv=0)), (UNS, dict(ldk=260)), (UNS, dict(ldv=257)),
    (INV, dict(seq=None)), (INV, dict(pos=None)), (INV, dict(k=None)), (INV, dict(v=None)), (UNS, dict(k=0x6008)),
    (UNS, dict(v=0x7002)), (OK, dict(rows=0, seq=None, k=None)), (OK, dict(cache=NOTHING))])
def test_rows_arguments(want, kw):
    assert _rows(**kw) == want


def _append(cfg=None, cache=None, **kw):
    a = {**dict(lens=0x5004, qkv=0x6000, ldqkv=1024, q=0x9000, ldq=512), **kw}
    return pp.lib().pp_paged_append(ctypes.byref(_cfg(**(cfg or {}))), ctypes.byref(_cache(**(cache or {}))), a["lens"],
                                    a["qkv"], a["ldqkv"], a["q"], a["ldq"], None)


@pytest.mark.parametrize("want,cfg,cache", CACHES + BUFFERS)
def test_append_cache(want, cfg, cache):
    assert _append(cfg, cache) == want


@pytest.mark.parametrize("want,kw", [
    (INV, dict(lens=None)), (INV, dict(qkv=None)), (INV, dict(q=None)), (INV, dict(ldqkv=1016)), (INV, dict(ldq=504)),
    (UNS, dict(ldqkv=1028)), (UNS, dict(ldq=513)), (UNS, dict(qkv=0x6008)), (UNS, dict(q=0x9004)),
    (INV, dict(q=0x6000)), (OK, dict(cache=NOTHING, lens=None))])
def test_append_arguments(want, kw):
    assert _append(**kw) == want


def _attend(cfg=None, cache=None, **kw):
    a = {**dict(lens=0x5004, q=0x6000, ldq=512, out=0x9000, ws=0x10000, bytes=1 << 40), **kw}
    return pp.lib().pp_paged_attention(ctypes.byref(_cfg(**(cfg or {}))), ctypes.byref(_cache(**(cache or {}))), a["lens"],
                                       a["q"], a["ldq"], a["out"], a["ws"], a["bytes"], None)


def _attend_bytes(cfg=None, cache=None):
    n = ctypes.c_size_t(7)
    st = pp.lib().pp_paged_attention_workspace_size(ctypes.byref(_cfg(**(cfg or {}))), ctypes.byref(_cache(**(cache or {}))),
                                                    ctypes.byref(n))
    return st, n.value


@pytest.mark.parametrize("want,cfg,cache", CACHES + BUFFERS)
def test_attention_cache(want, cfg, cache):
    assert _attend(cfg, cache) == want
    assert _attend_bytes(cfg, cache)[0] == (want if (want, cfg, cache) in CACHES else OK)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(lens=None)), (INV, dict(q=None)), (INV, dict(out=None)), (INV, dict(ldq=504)), (UNS, dict(ldq=516)),
    (UNS, dict(q=0x6004)), (UNS, dict(out=0x9008)), (OK, dict(cache=NOTHING, lens=None, ws=None, bytes=0))])
def test_attention_arguments(want, kw):
    assert _attend(**kw) == want


def test_attention_workspace():
    assert pp.lib().pp_paged_attention_workspace_size(ctypes.byref(_cfg()), ctypes.byref(_cache()), None) == INV
    for k in (1, 3, 64, 1000):
        st, need = _attend_bytes(cache=dict(k=k))
        assert st == OK and need <= 2048 * (2 * 4 * 4 * 136 + 32)
        if need:
            assert _attend(cache=dict(k=k), ws=None) == INV
            assert _attend(cache=dict(k=k), ws=0x10010) == INV
            assert _attend(cache=dict(k=k), bytes=need - 1) == SMALL


def _sample(**kw):
    a = {**dict(logits=0x1004, ldl=1000, k=3, vocab=1000, u=0x2004, ws=0x10000, bytes=1 << 40, tokens=0x3004), **kw}
    return pp.lib().pp_sample(a["logits"], a["ldl"], a["k"], a["vocab"], None, None, None, None, a["u"], a["ws"], a["bytes"],
                              a["tokens"], None, None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(k=-1)), (INV, dict(vocab=0)), (INV, dict(vocab=-5)), (INV, dict(ldl=999)), (INV, dict(logits=None)),
    (INV, dict(u=None)), (INV, dict(tokens=None)), (UNS, dict(vocab=1 << 20, ldl=1 << 21)), (UNS, dict(k=1 << 21)),
    (OK, dict(k=0, logits=None, u=None, tokens=None, ws=None, bytes=0))])
def test_sample_arguments(want, kw):
    assert _sample(**kw) == want


def test_sample_workspace():
    for k, vocab in [(1, 10), (1, 32000), (64, 128256), (300, 128256), (2, (1 << 20) - 1)]:
        need = pp.pp_sample_workspace_size(k, vocab)
        assert 0 <= need <= 1 << 26
        if need:
            kw = dict(k=k, vocab=vocab, ldl=vocab)
            assert _sample(ws=None, **kw) == INV
            assert _sample(ws=0x10010, **kw) == INV
            assert _sample(bytes=need - 1, **kw) == SMALL
    for vocab in (1000, 16384, 16385, 32000, 40000, 128256):    # the largest batch's workspace serves all
        sizes = [pp.pp_sample_workspace_size(k, vocab) for k in range(1, 1400)]
        assert sizes == sorted(sizes)
    for bad in [(-1, 10), (1, 0), (1, 1 << 20)]:
        with pytest.raises(pp.PrepackError):
            pp.pp_sample_workspace_size(*bad)
    assert pp.lib().pp_sample_workspace_size(1, 10, None) == INV


def test_paged_cache_tensors():
    """The binding takes tensors of the stated types and shapes only."""
    import torch
    assert ctypes.sizeof(pp.PPPagedCache) == 6 * 4 + 5 * 8     # 5 int32 + padding to 8 bytes
    table = torch.zeros((2, 3), dtype=torch.int32)
    pages = torch.zeros((5, 16, 256), dtype=torch.bfloat16)
    c = pp.PagedCache(pp.PP_KV_BF16, table, pages, pages.clone())
    assert (c.struct.k, c.struct.max_pages, c.struct.n_pages, c.struct.page_size) == (2, 3, 5, 16)
    codes, scale = torch.zeros((5, 16, 256), dtype=torch.int8), torch.zeros((5, 16, 2))
    pp.PagedCache(pp.PP_KV_I8, table, codes, codes, scale, scale)
    for bad in [(pp.PP_KV_F32, table, pages, pages), (pp.PP_KV_BF16, table.long(), pages, pages),
                (pp.PP_KV_BF16, table, pages, pages[:4]), (pp.PP_KV_I8, table, codes, codes),
                (pp.PP_KV_I8, table, codes, codes, scale, scale[:, :8]), (pp.PP_KV_BF16, table.t(), pages, pages),
                (pp.PP_KV_BF16, table, pages.transpose(0, 1), pages.transpose(0, 1))]:
        with pytest.raises(ValueError):
            pp.PagedCache(*bad)


# ----------------------------------------------------------------------------- index arithmetic
@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("paged") / "paged_index")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-I", os.path.join(ROOT, "paper_2404_09529_amd", "csrc"), os.path.join(ROOT, "tests", "host", "paged_index.cpp"),
                    "-o", exe], check=True, timeout=300)

    def f(lines):
        r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True, timeout=300)
        return [list(map(int, line.split())) for line in r.stdout.splitlines()]

    return f


def test_rows_of_pages(ask):
    """Rows stay inside the pool whatever the table holds, and pages that are not the pool's hold nothing."""
    rng = random.Random(1)
    cases = []
    for _ in range(200):
        shift, n_pages, max_pages = rng.randrange(0, 6), rng.randrange(1, 20), rng.randrange(0, 9)
        pages = [rng.choice([rng.randrange(n_pages), rng.randrange(n_pages), -1, n_pages, -2 ** 31, 2 ** 31 - 1]) for _ in range(max_pages)]
        cases.append((shift, n_pages, max_pages, pages))
    got = ask(["rows %d %d %d %s" % (n, s, m, " ".join(map(str, p))) for s, n, m, p in cases])
    for (shift, n_pages, max_pages, pages), g in zip(cases, got):
        span = max_pages << shift
        assert g[-3:] == [0, 0, span]
        want = [-1]
        for pos in range(span):
            page = pages[pos >> shift]
            want.append((page << shift) + pos % (1 << shift) if 0 <= page < n_pages else -1)
        assert g[:-3] == want + [-1, -1]
        assert all(-1 <= r < n_pages << shift for r in g[:-3])


def test_ranges_cover_every_step_once(ask):
    """Ranges follow one another from the first step to the last, differ by one step at most, and the joining kernel's
    view of a sequence, the ranges of its first and last step, is the ranges' own."""
    rng = random.Random(2)
    cases = [(16, [1]), (1, [5]), (7, [0, 0, 3]), (256, [100000, 0, 3]), (3, [2 ** 31 - 1] * 5), (16384, [2 ** 31 - 1] * 40)]
    for _ in range(150):
        top = rng.choice([1, 200, 5000, 100000])
        cases.append((rng.choice([1, 5, 16, 51, 256, 2048]), [rng.choice([0, rng.randrange(1, top + 1)]) for _ in range(rng.randrange(1, 40))] + [1]))
    got = ask(["split %d %s" % (w, " ".join(map(str, lens))) for w, lens in cases])
    for (W, lens), g in zip(cases, got):
        starts, ends = g[:W + 1], g[W + 2:]
        steps = [-(-n // 32) for n in lens if n]
        S = sum(steps)
        assert starts[0] == 0 and starts[W] == S and g[W + 1] == -1
        sizes = [b - a for a, b in zip(starts, starts[1:])]
        assert min(sizes) >= 0 and max(sizes) - min(sizes) <= 1
        at = 0
        for i, n in enumerate(steps):
            for s, r in ((at, ends[2 * i]), (at + n - 1, ends[2 * i + 1])):
                assert starts[r] <= s < starts[r + 1]
                assert S >= W or sizes[r] == 1
            at += n


@pytest.mark.parametrize("heads", [1, 2, 3, 8, 10, 32, 40, 64, 100, 257, 2048, 2049, 5000])
def test_every_range_and_head_has_a_wavefront(ask, heads):
    (got,) = ask(["places %d" % heads])
    groups, ranges, places = got[0], got[1], list(zip(got[2::2], got[3::2]))
    assert groups % 8 == 0 and ranges >= 1 and len(places) == groups * 8
    assert sorted(p for p in places if p[0] < ranges) == [(r, h) for r in range(ranges) for h in range(heads)]
