"""A paged cache on the GPU, through the C ABI, against float64 on the CPU.

Tolerances count roundings: half a step is 2^-24 of the value in float32 and 2^-8 in bf16."""
import math

import numpy as np
import pytest
import torch

from paper_2404_09529_amd import prepack as pp

from .gpu_util import require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": (pp.PP_BF16, torch.bfloat16), "f32": (pp.PP_F32, torch.float32)}
PAGES = {"f32": (pp.PP_KV_F32, torch.float32), "bf16": (pp.PP_KV_BF16, torch.bfloat16), "i8": (pp.PP_KV_I8, torch.int8)}
KINDS = [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "i8")]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def config(H, Hkv, D, dtype, theta=1e4):
    return pp.PPConfig(n_layers=1, d_model=256, n_heads=H, n_kv_heads=Hkv, head_dim=D, ffn_dim=256, vocab=1000,
                       dtype=TYPES[dtype][0], rms_eps=1e-5, rope_theta=theta)


def rand(g, *size):
    return torch.randn(size, generator=g)


class Pool:
    """Pages of one layer on the GPU with every row at a known value, sequences in shuffled pages."""

    def __init__(self, kv, k, Hkv, D, page, max_pages, spare=2, seed=0, fill=None):
        g = torch.Generator().manual_seed(seed)
        self.kv, self.Hkv, self.D, self.page = kv, Hkv, D, page
        n = k * max_pages + spare
        self.table = torch.randperm(n, generator=g)[:k * max_pages].view(k, max_pages).to(torch.int32)
        t = PAGES[kv][1]
        shape = (n, page, Hkv * D)
        if kv == "i8":
            self.k, self.v = (torch.full(shape, 55, dtype=t) for _ in range(2))
            self.ks, self.vs = (torch.full((n, page, Hkv), -3.0) for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, -7.0 if fill is None else fill, dtype=t) for _ in range(2))
            self.ks = self.vs = None
        self.to_device()

    def to_device(self):
        dev = [None if x is None else x.cuda() for x in (self.table, self.k, self.v, self.ks, self.vs)]
        self.cache = pp.PagedCache(PAGES[self.kv][0], *dev)
        self.dev = dict(zip(("table", "k", "v", "ks", "vs"), dev))
        return self

    def fill(self, seed, loud=1.0):
        """Every row a random one (8-bit pages: random codes and scales), on both sides."""
        g = torch.Generator().manual_seed(seed)
        if self.kv == "i8":
            for x in (self.k, self.v):
                x.copy_(torch.randint(-127, 128, x.shape, generator=g, dtype=torch.int8))
            for s in (self.ks, self.vs):
                s.copy_(torch.exp(0.5 * rand(g, *s.shape)) * loud / 70)
        else:
            self.k.copy_(rand(g, *self.k.shape) * loud)
            self.v.copy_(rand(g, *self.v.shape))
        return self.to_device()

    def row(self, i, pos):
        """Row of the pool, or None."""
        if not (0 <= i < self.table.shape[0] and 0 <= pos < self.table.shape[1] * self.page):
            return None
        p = int(self.table[i, pos // self.page])
        return p * self.page + pos % self.page if 0 <= p < self.k.shape[0] else None

    def host(self):
        """What the device holds now: k, v [rows, Hkv D] and the scales [rows, Hkv]."""
        k, v = (self.dev[n].cpu().view(-1, self.Hkv * self.D) for n in "kv")
        ks, vs = (None if self.dev[n] is None else self.dev[n].cpu().view(-1, self.Hkv) for n in ("ks", "vs"))
        return k, v, ks, vs

    def values(self):
        """k, v [rows, Hkv, D] in float64."""
        k, v, ks, vs = self.host()
        k, v = (x.double().view(-1, self.Hkv, self.D) for x in (k, v))
        return (k, v) if ks is None else (k * ks.double()[..., None], v * vs.double()[..., None])


def codes_of(x):
    """Codes and scales of float32 rows [..., D], by their definition."""
    x = x.float().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(x).max(-1)
        s = top * (np.float32(1) / np.float32(127))
        q = np.where(s[..., None] > 0, np.clip(np.rint(x / s[..., None]), -127, 127), 0)
    bad = ~np.isfinite(top)
    s[bad], q[bad] = np.nan, 0
    return torch.from_numpy(q).to(torch.int8), torch.from_numpy(s)


# ----------------------------------------------------------------------------- rows in and out
ROWS = [  # H, Hkv, D of a config, page size, rows
    ("bf16", 2, 2, 128, 16, 1), ("bf16", 4, 2, 128, 1, 37), ("bf16", 8, 8, 128, 64, 700), ("f32", 1, 1, 64, 4, 5),
    ("f32", 6, 2, 64, 32, 250), ("f32", 5, 5, 128, 8, 131)]


@pytest.mark.parametrize("dtype,H,Hkv,D,page,rows", ROWS)
@pytest.mark.parametrize("eight", [False, True])
def test_write_then_read(dtype, H, Hkv, D, page, rows, eight):
    """Strided rows to shuffled places, some without one; everything else stays as it was."""
    kv, t = "i8" if eight else dtype, TYPES[dtype][1]
    g = torch.Generator().manual_seed(rows)
    k, kvw = 3, Hkv * D
    pool = Pool(kv, k, Hkv, D, page, -(-rows // page) + 1, seed=rows)
    pool.table[1, 0], pool.table[2, 0] = -1, pool.k.shape[0]
    pool.to_device()
    places = [(i, j) for i in range(-1, k + 1) for j in range(-2, pool.table.shape[1] * page + 2)]
    places = [places[j] for j in torch.randperm(len(places), generator=g)[:rows].tolist()]
    seq, pos = (torch.tensor(x, dtype=torch.int32).cuda() for x in zip(*places))
    ldk, ldv = kvw + 16, kvw + 8
    keys, values = (rand(g, rows, ld) * torch.exp(2 * rand(g, rows, 1)) for ld in (ldk, ldv))
    keys, values = keys.to(t), values.to(t)
    cfg = config(H, Hkv, D, dtype)
    want_k, want_v, want_ks, want_vs = pool.host()
    pp.pp_paged_write(cfg, pool.cache, seq, pos, rows, keys.cuda(), ldk, values.cuda(), ldv)
    for r, (i, j) in enumerate(places):
        at = pool.row(i, j)
        if at is None:
            continue
        for x, pages, scales in ((keys[r, :kvw], want_k, want_ks), (values[r, :kvw], want_v, want_vs)):
            if eight:
                q, s = codes_of(x.view(Hkv, D))
                pages[at], scales[at] = q.view(-1), s
            else:
                pages[at] = x
    for got, want in zip(pool.host(), (want_k, want_v, want_ks, want_vs)):
        assert want is None or torch.equal(got, want)
    # and back: the code's product with its scale, rounded once; rows without a place are left alone
    out_k, out_v = torch.full((rows + 1, ldv), 9.0).to(t).cuda(), torch.full((rows + 1, ldk), 9.0).to(t).cuda()
    pp.pp_paged_read(cfg, pool.cache, seq, pos, rows, out_k, ldv, out_v, ldk)
    for out, ld, pages, scales in ((out_k, ldv, want_k, want_ks), (out_v, ldk, want_v, want_vs)):
        want = torch.full((rows + 1, ld), 9.0).to(t)
        for r, (i, j) in enumerate(places):
            at = pool.row(i, j)
            if at is not None:
                x = pages[at].float().view(Hkv, D) * scales[at][:, None] if eight else pages[at].view(Hkv, D)
                want[r, :kvw] = x.reshape(-1).to(t)
        assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write_special_rows(dtype):
    """Zeros, the type's largest values, denormals, ties, NaN and infinities in 8 bits."""
    D, t = 128, TYPES[dtype][1]
    x = torch.zeros(10, D)
    x[1, 3], x[1, 4] = 3e38, -3e38
    x[2, 0] = 1e-40
    x[3] = torch.linspace(-1.2e-38, 1.2e-38, D)
    x[4, :4] = torch.tensor([127.0, 0.5, 1.5, -2.5])
    x[5, 7] = float("nan")
    x[6, 9] = float("inf")
    x[7, 1] = -float("inf")
    x[8] = -0.0
    x[9] = 1e-45
    x = x.to(t)
    pool = Pool("i8", 1, 1, D, 16, 1)
    at = torch.arange(10, dtype=torch.int32).cuda()
    cfg = config(2, 1, D, dtype) if dtype == "f32" else config(6, 1, D, dtype)
    pp.pp_paged_write(cfg, pool.cache, torch.zeros_like(at), at, 10, x.cuda(), D, x.flip(0).contiguous().cuda(), D)
    k, v, ks, vs = pool.host()
    rows = [pool.row(0, j) for j in range(10)]
    for y, codes, scales in ((x, k, ks), (x.flip(0), v, vs)):
        q, s = codes_of(y)
        assert torch.equal(codes[rows], q) and torch.equal(scales[rows][:, 0].nan_to_num(5.0), s.nan_to_num(5.0))
    out = [torch.empty(10, D, dtype=t, device="cuda") for _ in range(2)]
    pp.pp_paged_read(cfg, pool.cache, torch.zeros_like(at), at, 10, out[0], D, out[1], D)
    assert out[0][5:8].isnan().all() and out[0][[0, 1, 2, 3, 4, 8, 9]].isfinite().all()


# ----------------------------------------------------------------------------- append
HEADS = [("bf16", 2, 1, 128), ("bf16", 8, 8, 128), ("bf16", 32, 8, 128), ("f32", 1, 1, 64), ("f32", 6, 3, 64),
         ("f32", 9, 3, 128)]


def rotated(x, pos, theta):
    """Heads [.., D] in float64 rotated by position pos: cosines and sines are float32 numbers."""
    half = x.shape[-1] // 2
    angle = pos * theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / (2 * half))
    c, s = angle.cos().float().double(), angle.sin().float().double()
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


@pytest.mark.parametrize("dtype,H,Hkv,D", [h for h in HEADS if h[0] == "f32" or (h[1] + 2 * h[2]) % 2 == 0])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_append(dtype, H, Hkv, D, eight, in_place):
    kv, t, theta = "i8" if eight else dtype, TYPES[dtype][1], 5e5
    page, lens = 8, [1, 0, 8, 9, -4, 33, 40, 41, 2 ** 31 - 1]   # the last two are past the table
    k, w = len(lens), (H + 2 * Hkv) * D
    pool = Pool(kv, k, Hkv, D, page, 5, seed=3)
    pool.table[5, 4] = -1                                       # position 32 has no page
    pool.to_device()
    g = torch.Generator().manual_seed(H)
    ld = w + 24
    qkv = (rand(g, k, ld) * torch.exp(rand(g, k, 1))).to(t)
    dev = qkv.cuda()
    ldq = ld if in_place else H * D + 8
    q_out = dev if in_place else torch.full((k + 1, ldq), 9.0).to(t).cuda()
    before = q_out.cpu()
    want = pool.host()
    pp.pp_paged_append(config(H, Hkv, D, dtype, theta), pool.cache, torch.tensor(lens, dtype=torch.int32).cuda(), dev, ld, q_out, ldq)
    got, got_q = pool.host(), q_out.cpu()
    for i, n in enumerate(lens):
        if n <= 0:
            assert torch.equal(got_q[i], before[i])
            continue
        x = qkv[i, :w].double().view(H + 2 * Hkv, D)
        turned = rotated(x[:H + Hkv], n - 1, theta)
        # the angle is off by 2 float64 steps of itself, an entry by that and, next to a border, a float32 step
        entry = 2.0 * U + n * 2.0 ** -50
        size = x[:H + Hkv].abs() + x[:H + Hkv].roll(D // 2, -1).abs()
        off = size * entry + turned.abs() * 1.01 * U + 1e-37
        tol = off + (turned.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
        assert torch.all((got_q[i, :H * D].double().view(H, D) - turned[:H]).abs() <= tol[:H])
        assert torch.equal(got_q[i, H * D:], before[i, H * D:])
        at = pool.row(i, n - 1)
        if at is None:
            continue
        value = x[H + Hkv:]
        if eight:
            q, s = codes_of(value.float())
            assert torch.equal(got[1][at].view(Hkv, D), q) and torch.equal(got[3][at], s)
            key, key_off, scale = turned[H:], off[H:], got[2][at].double()
            top = key.abs().amax(1)
            assert torch.all((scale - top / 127).abs() <= key_off.amax(1) / 127 + 2.01 * U * top / 127)
            live = scale[:, None]
            code = got[0][at].double().view(Hkv, D)
            assert torch.all((code - key / live).abs() <= 0.5 + key_off / live + 127.1 * 4 * U) and code.abs().max() <= 127
        else:
            assert torch.equal(got[1][at].view(Hkv, D), value.to(t))
            assert torch.all((got[0][at].double().view(Hkv, D) - turned[H:]).abs() <= tol[H:])
        for w_, g_ in zip(want, got):                          # what the comparison below leaves out
            if w_ is not None:
                w_[at] = g_[at]
    for w_, g_ in zip(want, got):
        assert w_ is None or torch.equal(w_, g_)
    if not in_place:
        assert torch.equal(got_q[k], before[k]) and torch.equal(dev.cpu(), qkv)


# ----------------------------------------------------------------------------- attention
def attention64(q, pool, lens, H):
    """out [k, H, D] in float64, and the tolerance's ingredients: sum |q_d k_d| of the largest score, and sum p |v|."""
    Hkv, D = pool.Hkv, pool.D
    K, V = pool.values()
    out, size, vabs = torch.zeros(len(lens), H, D, dtype=torch.float64), torch.zeros(len(lens), H, 1, dtype=torch.float64), torch.zeros(len(lens), H, D, dtype=torch.float64)
    for i, n in enumerate(lens):
        rows = [pool.row(i, j) for j in range(min(max(n, 0), pool.table.shape[1] * pool.page))]
        rows = [r for r in rows if r is not None]
        if not rows:
            continue
        for h in range(H):
            kk, vv, x = K[rows, h // (H // Hkv)], V[rows, h // (H // Hkv)], q[i, h]
            s = (kk * x).sum(1) / math.sqrt(D)
            p = torch.softmax(s, 0)
            out[i, h] = (p[:, None] * vv).sum(0)
            size[i, h] = (kk.abs() * x.abs()).sum(1).max() / math.sqrt(D)
            vabs[i, h] = (p[:, None] * vv.abs()).sum(0)
    return out, size, vabs


def run_attention(cfg, pool, lens, q, ldq=None, out=None, stream=None):
    k, w = len(lens), cfg.n_heads * cfg.head_dim
    t = q.dtype
    out = torch.full((k + 1, w), 9.0, device="cuda").to(t) if out is None else out
    need = pp.pp_paged_attention_workspace_size(cfg, pool.cache)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")    # NaN as float32
    dev = torch.tensor(lens, dtype=torch.int32).cuda()
    pp.pp_paged_attention(cfg, pool.cache, dev, q, w if ldq is None else ldq, out, ws[:need], stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 255).all())
    return out


def check_attention(got, q, pool, lens, H, dtype):
    """A score is a sum of D products and up to three more roundings, each at most (D + 3) 2^-24 of the sum of the products'
    sizes; the exponential's argument and value add 2^-24 of the score and 4 steps.  A relative change by e of the
    probabilities changes the result by 2 e sum p |v|.  The sums over n keys add (n + 8) 2^-24 of sum p |v|, and probabilities
    may be fed to the matrix cores as two bf16 terms, 2^-16.  bf16 results are rounded once, 2^-8."""
    want, size, vabs = attention64(q, pool, lens, H)
    n = torch.tensor([min(max(x, 0), pool.table.shape[1] * pool.page) for x in lens], dtype=torch.float64)[:, None, None]
    e = (pool.D + 6) * U * size + 8 * U + (2.0 ** -16 if dtype == "bf16" else 0)
    tol = (2 * e + (n + 8) * U) * vabs + 1e-37
    if dtype == "bf16":
        tol = tol + (want.abs() + tol) * 2.0 ** -8
    err = (got[:len(lens)].double().cpu().view(want.shape) - want).abs()
    worst = float((err / tol).max())
    print(f"[paged attention] worst error / tolerance {worst:.3f}", flush=True)
    assert worst <= 1.0
    assert bool((got[len(lens):].float() == 9.0).all())


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500, 1023, 1111]
ATTENTION = [  # H, Hkv, D
    ("bf16", 2, 2, 128), ("bf16", 8, 4, 128), ("bf16", 12, 2, 128), ("bf16", 16, 1, 128), ("bf16", 20, 1, 128),
    ("bf16", 40, 1, 128), ("bf16", 32, 8, 128), ("f32", 1, 1, 64), ("f32", 4, 2, 64), ("f32", 3, 3, 128), ("f32", 8, 1, 128),
    ("f32", 17, 1, 64), ("f32", 10, 2, 128)]


@pytest.mark.parametrize("page", [1, 4, 16, 256])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,H,Hkv,D", ATTENTION)
def test_attention(dtype, H, Hkv, D, eight, page):
    """Many lengths at once, sharp scores, strided queries."""
    kv, t = "i8" if eight else dtype, TYPES[dtype][1]
    pool = Pool(kv, len(LENS), Hkv, D, page, -(-1111 // page), seed=page).fill(H)
    g = torch.Generator().manual_seed(H + page)
    ldq = H * D + 40
    q = (2.0 * rand(g, len(LENS), ldq)).to(t)
    got = run_attention(config(H, Hkv, D, dtype), pool, LENS, q.cuda(), ldq)
    check_attention(got, q[:, :H * D].double().view(-1, H, D), pool, LENS, H, dtype)


@pytest.mark.parametrize("dtype,kv", KINDS)
@pytest.mark.parametrize("lens", [[1], [33], [5000], [20011], [7000, 1, 0, 12345], [1] * 300, [0, 0, 0], [260] * 70])
def test_attention_splits(dtype, kv, lens):
    """One long sequence alone, long ones among short ones, more sequences than workgroups."""
    H, Hkv, D = (8, 2, 128) if dtype == "bf16" else (4, 2, 64)
    pool = Pool(kv, len(lens), Hkv, D, 32, -(-max(max(lens), 1) // 32), seed=len(lens)).fill(len(lens))
    g = torch.Generator().manual_seed(7)
    q = (2.0 * rand(g, len(lens), H * D)).to(TYPES[dtype][1])
    cfg = config(H, Hkv, D, dtype)
    got = run_attention(cfg, pool, lens, q.cuda())
    check_attention(got, q.double().view(-1, H, D), pool, lens, H, dtype)
    assert torch.equal(run_attention(cfg, pool, lens, q.cuda()), got)      # deterministic


@pytest.mark.parametrize("dtype,kv", KINDS)
def test_attention_places_that_hold_nothing(dtype, kv):
    """Lengths below zero and past the table, pages that are not the pool's: at the start, inside a tile, everywhere;
    what lies in rows that no sequence reaches does not matter, NaN and infinities included."""
    H, Hkv, D = (6, 1, 128) if dtype == "bf16" else (6, 2, 64)
    lens = [-5, 300, 2 ** 31 - 1, 70, 129, 200, 40, 3]
    pool = Pool(kv, len(lens), Hkv, D, 4, 64, seed=9).fill(1)
    n = pool.k.shape[0]
    pool.table[1, 3:5] = -1                                    # inside a tile
    pool.table[2, 40] = n                                      # the first id past the pool
    pool.table[3, :] = torch.tensor([-1, n, -2 ** 31, 2 ** 31 - 1]).repeat(16).to(torch.int32)   # nothing at all
    pool.table[4, :32] = -7                                    # all of the first tile: one key is left
    pool.table[5, 1:] = 2 ** 30                                # the first page only
    pool.table[6, 9] = -1                                      # the last page
    used = {pool.row(i, j) for i, m in enumerate(lens) for j in range(min(max(m, 0), 256))} - {None}
    free = torch.tensor(sorted(set(range(n * 4)) - used))
    for x, s in ((pool.k, pool.ks), (pool.v, pool.vs)):
        bad = torch.tensor([float("nan"), float("inf"), -float("inf")])[torch.arange(free.numel()) % 3]
        if kv == "i8":
            s.view(-1, Hkv)[free] = bad[:, None]
        else:
            x.view(-1, Hkv * D)[free] = bad[:, None].to(x.dtype)
    pool.to_device()
    q = (2.0 * rand(torch.Generator().manual_seed(2), len(lens), H * D)).to(TYPES[dtype][1])
    got = run_attention(config(H, Hkv, D, dtype), pool, lens, q.cuda())
    check_attention(got, q.double().view(-1, H, D), pool, lens, H, dtype)
    assert bool((got[[0, 3]] == 0).all())


@pytest.mark.parametrize("dtype,kv", KINDS)
@pytest.mark.parametrize("lens", [[700, 300, 140], [9000, 300, 140]])
def test_attention_special_values(dtype, kv, lens):
    """NaN in a key reaches the heads that read it and no others; scores of -inf count nothing beside others
    and are not a number alone; the largest finite scores are scores."""
    H, Hkv, D = (4, 2, 128) if dtype == "bf16" else (4, 2, 64)
    t = TYPES[dtype][1]
    pool = Pool(kv, 3, Hkv, D, 16, -(-max(lens) // 16), seed=4).fill(5)
    q = rand(torch.Generator().manual_seed(3), 3, H, D)
    q[1, 0] = torch.finfo(t).max                               # head 0 of sequence 1: products overflow
    where = pool.row(0, 77)
    if kv == "i8":
        pool.ks.view(-1, Hkv)[where, 1] = float("nan")
    else:
        pool.k.view(-1, Hkv, D)[where, 1, 5] = float("nan")
        q[2, 1] = 0.0
        q[2, 1, 0] = 1.0                                       # head 1 of sequence 2 reads element 0 of its keys
        rows = [pool.row(2, j) for j in range(140)]
        pool.k.view(-1, Hkv, D)[rows, 0, 0] = -float("inf")
        pool.k.view(-1, Hkv, D)[rows[:70] + rows[71:], 0, 0] = torch.finfo(t).min if dtype == "f32" else -float("inf")
        pool.k.view(-1, Hkv, D)[rows[70], 0, 0] = torch.finfo(t).min
    pool.to_device()
    q = q.to(t)
    got = run_attention(config(H, Hkv, D, dtype), pool, lens, q.view(3, -1).cuda()).float().cpu()[:3].view(3, H, D)
    assert got[0, 2:].isnan().all() and got[0, :2].isfinite().all()
    assert got[1, 1:].isfinite().all()
    if kv != "i8":
        rows = [pool.row(2, j) for j in range(140)]
        v = pool.v.view(-1, Hkv, D)[rows, 0].double()
        # keys of the type's lowest value among others of -inf, or all of them the same: products are exact
        want = v[70] if dtype == "bf16" else v.mean(0)
        if dtype == "bf16":
            assert torch.all((got[2, 1].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -15))
        else:
            assert torch.all((got[2, 1].double() - want).abs() <= 160 * U * v.abs().mean(0))
        pool.k.view(-1, Hkv, D)[rows, 0, 0] = -float("inf")    # nothing but -inf
        pool.to_device()
        got = run_attention(config(H, Hkv, D, dtype), pool, lens, q.view(3, -1).cuda()).float().cpu()[2].view(H, D)
        assert got[1].isnan().all() and got[2:].isfinite().all()


@pytest.mark.parametrize("kv", ["bf16", "i8"])
def test_pool_past_32_bits(kv):
    """Rows beyond 2^32 bytes (and elements) of the pool, by all four calls."""
    H, Hkv, D, page = 32, 32, 128, 64
    kvw = Hkv * D
    n_pages = (2 ** 32 // kvw // page) + 5 if kv == "i8" else (2 ** 32 // kvw // page) // 2 + 5
    t, code = torch.bfloat16, PAGES[kv]
    k, v = (torch.zeros((n_pages, page, kvw), dtype=code[1], device="cuda") for _ in range(2))
    scales = [torch.zeros((n_pages, page, Hkv), device="cuda") for _ in range(2)] if kv == "i8" else [None, None]
    last = list(range(n_pages - 1, n_pages - 4, -1))
    table = torch.tensor([last, [0, n_pages - 4, 1]], dtype=torch.int32, device="cuda")
    cache = pp.PagedCache(code[0], table, k, v, *scales)
    cfg = config(H, Hkv, D, "bf16")
    n = 150
    g = torch.Generator(device="cuda").manual_seed(1)
    keys, values = (torch.randn((2 * n, kvw), generator=g, device="cuda").to(t) for _ in range(2))
    seq = torch.tensor([0] * n + [1] * n, dtype=torch.int32, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda").repeat(2)
    pp.pp_paged_write(cfg, cache, seq, pos, 2 * n, keys, kvw, values, kvw)
    lens = torch.tensor([n + 1, n + 1], dtype=torch.int32, device="cuda")
    qkv = torch.randn((2, 3 * kvw), generator=g, device="cuda").to(t)
    q = torch.empty((2, kvw), dtype=t, device="cuda")
    pp.pp_paged_append(cfg, cache, lens, qkv, 3 * kvw, q, kvw)
    seq, pos = torch.tensor([0] * (n + 1) + [1] * (n + 1), dtype=torch.int32, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda").repeat(2)
    bk, bv = (torch.empty((2 * n + 2, kvw), dtype=t, device="cuda") for _ in range(2))
    pp.pp_paged_read(cfg, cache, seq, pos, 2 * n + 2, bk, kvw, bv, kvw)
    bk, bv = bk.cpu().view(2, n + 1, Hkv, D).double(), bv.cpu().view(2, n + 1, Hkv, D).double()
    want_k, want_v = keys.cpu().view(2, n, Hkv, D).double(), values.cpu().view(2, n, Hkv, D).double()
    step = 2.0 ** -8 if kv == "i8" else 0.0     # rounding of the value read
    half = (lambda x: x.abs().amax(-1, keepdim=True) / 127 * 0.5001) if kv == "i8" else (lambda x: 0 * x)
    for got, want in ((bk[:, :n], want_k), (bv[:, :n], want_v), (bv[:, n], qkv[:, 2 * kvw:].cpu().view(2, Hkv, D).double())):
        assert torch.all((got - want).abs() <= half(want) + step * (want.abs() + half(want)))
    out = torch.empty((2, kvw), dtype=t, device="cuda")
    ws = torch.empty(max(pp.pp_paged_attention_workspace_size(cfg, cache), 1), dtype=torch.uint8, device="cuda")
    pp.pp_paged_attention(cfg, cache, lens, q, kvw, out, ws)
    if kv == "i8":                              # the attention reads codes; these are the values in full
        flat = [(x.view(-1, Hkv, D), s.view(-1, Hkv)) for x, s in ((k, scales[0]), (v, scales[1]))]
        rows = [[int(table[i, j // page]) * page + j % page for j in range(n + 1)] for i in range(2)]
        bk, bv = (torch.stack([x[r].double().cpu() * s[r].double().cpu()[..., None] for r in rows]) for x, s in flat)
    s = (bk * q.cpu().view(2, 1, H, D).double()).sum(-1) / math.sqrt(D)
    p = torch.softmax(s, 1)[..., None]
    want = (p * bv).sum(1)
    tol = (p * bv.abs()).sum(1) * 2.0 ** -14 + want.abs() * 2.0 ** -8
    assert torch.all((out.cpu().double().view(2, H, D) - want).abs() <= tol)


@pytest.mark.parametrize("dtype,kv", KINDS)
def test_decode_step_in_a_graph(dtype, kv):
    """append and attention recorded once and replayed while lengths and pages change, a second graph with a workspace
    of its own in between; every replay equals the eager calls."""
    H, Hkv, D = (6, 2, 128) if dtype == "bf16" else (4, 2, 64)
    t, w = TYPES[dtype][1], (H + 2 * Hkv) * D
    cfg, k = config(H, Hkv, D, dtype), 5
    lens0 = [1, 15, 16, 300, 0]
    pools = [Pool(kv, k, Hkv, D, 16, 24, seed=6).fill(8) for _ in range(2)]
    g = torch.Generator().manual_seed(5)
    steps = [rand(g, k, w).to(t) for _ in range(6)]
    ws = [torch.empty(max(pp.pp_paged_attention_workspace_size(cfg, p.cache), 1), dtype=torch.uint8, device="cuda") for p in pools]
    lens = [torch.tensor(lens0, dtype=torch.int32, device="cuda") for _ in pools]
    qkv = [steps[0].cuda() for _ in pools]
    q = [torch.zeros(k, H * D, dtype=t, device="cuda") for _ in pools]
    out = [torch.zeros(k, H * D, dtype=t, device="cuda") for _ in pools]

    def step(a):
        pp.pp_paged_append(cfg, pools[a].cache, lens[a], qkv[a], w, q[a], H * D)
        pp.pp_paged_attention(cfg, pools[a].cache, lens[a], q[a], H * D, out[a], ws[a])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(1)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            step(1)
    for n, x in enumerate(steps):
        for a in range(2):
            qkv[a].copy_(x)
            lens[a].copy_(torch.tensor([m + 17 * n if m else 0 for m in lens0], dtype=torch.int32))
        step(0)
        torch.cuda.synchronize()
        graphs[n % 2].replay()
        (out[0] + 1).sum()                                     # eager work beside it
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and torch.equal(q[0], q[1])
        for x0, x1 in zip(pools[0].host(), pools[1].host()):
            assert x0 is None or torch.equal(x0, x1)


def test_two_streams_at_once():
    """Calls on two streams with a workspace each; a call on a stream that is not the current one."""
    H, Hkv, D = 32, 8, 128
    cfg = config(H, Hkv, D, "bf16")
    lens = [3000, 17, 900, 1]
    pools = [Pool("bf16", 4, Hkv, D, 16, 190, seed=s).fill(s) for s in (1, 2)]
    q = [rand(torch.Generator().manual_seed(s), 4, H * D).bfloat16().cuda() for s in (1, 2)]
    want = [run_attention(cfg, p, lens, x) for p, x in zip(pools, q)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    dev = torch.tensor(lens, dtype=torch.int32).cuda()
    ws = [torch.empty(pp.pp_paged_attention_workspace_size(cfg, p.cache) + 1, dtype=torch.uint8, device="cuda") for p in pools]
    out = [torch.empty(4, H * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for a in range(2):
            pp.pp_paged_attention(cfg, pools[a].cache, dev, q[a], H * D, out[a], ws[a], stream=streams[a])
    torch.cuda.synchronize()
    for a in range(2):
        assert torch.equal(out[a], want[a][:4])


def test_shared_pages():
    """Two sequences with a common beginning in the same pages, which neither writes."""
    H, Hkv, D = 6, 2, 64
    pool = Pool("f32", 2, Hkv, D, 8, 10, seed=1).fill(1)
    pool.table[1, :4] = pool.table[0, :4]
    pool.to_device()
    lens = [60, 45]
    q = rand(torch.Generator().manual_seed(1), 2, H * D)
    got = run_attention(config(H, Hkv, D, "f32"), pool, lens, q.cuda())
    check_attention(got, q.double().view(2, H, D), pool, lens, H, "f32")


def _many(name):
    """Lengths of more sequences than a wavefront's registers hold at once (256), with empty ones around that border."""
    g = torch.Generator().manual_seed(11)
    n = torch.tensor([0, 1, 33, 70])[torch.randint(0, 4, (700,), generator=g)].tolist()
    if name == "border":
        n[250:259] = [0] * 9
        n[511:515] = [40, 0, 0, 0]
        n[249] = n[259] = 5
    elif name == "one before":
        n[254:258] = [33, 0, 20, 0]
    elif name == "gap of a block":
        n[200:600] = [0] * 400
    elif name == "late":
        n[:680] = [0] * 680
    elif name == "last alone":
        n = [0] * 699 + [50]
    elif name == "long":
        n[255], n[256], n[600] = 3000, 0, 4000
    return n


@pytest.mark.parametrize("dtype,kv", KINDS)
@pytest.mark.parametrize("name", ["random", "border", "one before", "gap of a block", "late", "last alone", "long"])
def test_attention_many_sequences(dtype, kv, name):
    lens = _many(name)
    H, Hkv, D = (2, 1, 128) if dtype == "bf16" else (1, 1, 64)
    pool = Pool(kv, len(lens), Hkv, D, 32, -(-max(lens) // 32), seed=3).fill(4)
    q = (2.0 * rand(torch.Generator().manual_seed(7), len(lens), H * D)).to(TYPES[dtype][1])
    got = run_attention(config(H, Hkv, D, dtype), pool, lens, q.cuda())
    check_attention(got, q.double().view(-1, H, D), pool, lens, H, dtype)


@pytest.mark.parametrize("kv", ["f32", "i8"])
def test_attention_tables_past_31_bits_of_steps(kv):
    """Tables that reach 2^31 - 1 positions each: 33 sequences' steps pass 2^31.  One sequence is that long, with one page."""
    H, Hkv, D, page, k = 2, 1, 64, 1 << 16, 33
    max_pages = (1 << 31) // page
    pool = Pool(kv, 1, Hkv, D, page, 1, spare=0, seed=3).fill(4)
    lens = [(i * 37) % 300 for i in range(k)]
    lens[3] = 2 ** 31 - 1
    table = torch.full((k, max_pages), -1, dtype=torch.int32)
    table[:, 0] = 0
    table[3, 0], table[3, max_pages - 1] = -1, 0        # the last page, but for the last position
    table[5, 0] = -1
    pool.table = table
    pool.to_device()
    q = (2.0 * rand(torch.Generator().manual_seed(7), k, H * D))
    got = run_attention(config(H, Hkv, D, "f32"), pool, lens, q.cuda())
    # the same keys for a table of one page
    pool.table, short = torch.zeros((k, 1), dtype=torch.int32), list(lens)
    pool.table[5, 0] = -1
    short[3] = page - 1
    pool.to_device()
    check_attention(got, q.double().view(-1, H, D), pool, short, H, "f32")


@pytest.mark.parametrize("dtype,kv", KINDS)
def test_tables_without_entries(dtype, kv):
    """max_pages 0: nothing has a place, the query is rotated all the same."""
    H, Hkv, D = (2, 1, 128) if dtype == "bf16" else (2, 1, 64)
    t, w, cfg = TYPES[dtype][1], (H + 2 * Hkv) * D, config(H, Hkv, D, dtype)
    pool = Pool(kv, 3, Hkv, D, 8, 1, seed=1).fill(2)
    before = pool.host()
    full = pool.cache
    dev = pool.dev
    cache = pp.PagedCache(PAGES[kv][0], torch.empty((3, 0), dtype=torch.int32, device="cuda"), dev["k"], dev["v"], dev["ks"], dev["vs"])
    qkv = rand(torch.Generator().manual_seed(3), 3, w).to(t).cuda()
    lens = torch.tensor([5, 0, 1], dtype=torch.int32, device="cuda")
    q, q2 = (torch.full((3, H * D), 9.0, device="cuda").to(t) for _ in range(2))
    pp.pp_paged_append(cfg, cache, lens, qkv, w, q, H * D)
    rows = torch.zeros(3, dtype=torch.int32, device="cuda")
    dense = torch.full((3, Hkv * D), 4.0, device="cuda").to(t)
    pp.pp_paged_write(cfg, cache, rows, rows, 3, dense, Hkv * D, dense, Hkv * D)
    pp.pp_paged_read(cfg, cache, rows, rows, 3, dense, Hkv * D, dense, Hkv * D)
    out = torch.full((3, H * D), 9.0, device="cuda").to(t)
    ws = torch.empty(pp.pp_paged_attention_workspace_size(cfg, cache), dtype=torch.uint8, device="cuda")
    pp.pp_paged_attention(cfg, cache, lens, q, H * D, out, ws)
    torch.cuda.synchronize()
    for x, y in zip(before, pool.host()):
        assert x is None or torch.equal(x, y)
    assert bool((dense == 4).all()) and bool((out == 0).all()) and bool((q[1] == 9).all())
    pp.pp_paged_append(cfg, full, lens, qkv, w, q2, H * D)
    torch.cuda.synchronize()
    assert torch.equal(q, q2)
