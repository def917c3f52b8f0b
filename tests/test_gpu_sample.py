"""pp_sample on the GPU against its definition in numpy with exact integer sums."""
import math

import numpy as np
import pytest
import torch

from paper_2404_09529_amd import prepack as pp

from .gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def definition(x, t=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, share) of one row, and whether a bound lies within a rounding of a place (then another token next to it in
    the order would do as well).  Weights are float64 exponentials, off by a few steps of 2^-53 in both computations, and
    multiples of 2^-44: a running sum is off by 2^-44 an id."""
    x = np.asarray(x, dtype=np.float32)
    ids = np.flatnonzero(~np.isnan(x))
    if not t > 0:
        return (int(ids[np.argmax(x[ids])]), 1.0, False) if ids.size else (-1, 0.0, False)
    ids = ids[x[ids] > -np.inf]
    if ids.size == 0:
        return -1, 0.0, False
    order = ids[np.argsort(-x[ids].astype(np.float64), kind="stable")]
    y = x[order].astype(np.float64)
    with np.errstate(invalid="ignore"):
        w = np.where(y == y[0], 1.0, np.exp((y - y[0]) / np.float64(np.float32(t)))) if np.isfinite(y[0]) else (y == y[0]).astype(np.float64)
    f = np.rint(w * 2.0 ** 44).astype(np.int64).astype(object) if w.size < 50 else np.rint(w * 2.0 ** 44).astype(np.int64)
    slack = 4.0 * len(f)
    n = int((np.asarray(f, dtype=np.float64) >= 1).sum())
    f, w, order = f[:n], w[:n], order[:n]
    cum = np.asarray(np.cumsum(f), dtype=np.float64)
    near = False
    kept = n if top_k <= 0 else min(n, top_k)
    if top_p < 1:
        bound = max(float(np.float32(top_p)) * cum[kept - 1], 1.0)
        place = int(np.argmax(cum[:kept] >= bound))
        near |= bool(np.min(np.abs(cum[:kept] - bound)) <= slack) and top_p > 0
        kept = place + 1
    if min_p > 0:
        m = min(float(np.float32(min_p)), 1.0)
        near |= bool(np.any(np.abs(w - m) <= 2.0 ** -50) and m < 1)
        kept = min(kept, int((w >= m).sum()))
    total = cum[kept - 1]
    uu = float(np.float32(u))
    uu = uu if uu >= 0 else 0.0                                # NaN too
    bound = uu * total if uu < 1 else total
    bound = min(bound, np.nextafter(total, 0))
    place = int(np.argmax(cum[:kept] > bound))
    near |= bool(np.min(np.abs(cum[:kept] - bound)) <= slack) and 0 < uu < 1
    # weights of 1 are exact in every computation, and so are their sums
    return int(order[place]), float(w[place] * 2.0 ** 44 / total), near and not bool((w == 1).all())


def run(x, t=None, top_k=None, top_p=None, min_p=None, u=None, ldl=None, stream=None):
    """x float32 [k, ldl]; settings lists or None."""
    k = x.shape[0]
    vocab = x.shape[1] if ldl is None else ldl
    f = lambda v, dt=torch.float32: None if v is None else torch.tensor(v, dtype=dt, device="cuda")
    tokens = torch.full((k + 1,), -9, dtype=torch.int32, device="cuda")
    prob = torch.full((k + 1,), -9.0, device="cuda")
    need = pp.pp_sample_workspace_size(k, vocab)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    pp.pp_sample(x.cuda(), x.shape[1], k, vocab, f(t), f(top_k, torch.int32), f(top_p), f(min_p), f(u), tokens, ws[:need], prob, stream)
    torch.cuda.synchronize()
    assert int(tokens[k]) == -9 and float(prob[k]) == -9.0 and bool((ws[need:] == 255).all())
    return tokens[:k].cpu().tolist(), prob[:k].cpu().double().tolist()


def check(x, vocab=None, **settings):
    """Every row against the definition; a share is off by its float32 rounding and by the weights' steps."""
    tokens, probs = run(x, ldl=vocab, **settings)
    xs, nears = x[:, :vocab].numpy(), 0
    for i in range(x.shape[0]):
        mine = {n: settings[n][i] for n in ("t", "top_k", "top_p", "min_p", "u") if settings.get(n) is not None}
        token, share, near = definition(xs[i], **mine)
        if near:
            nears += 1
            continue
        assert tokens[i] == token, (i, mine)
        assert abs(probs[i] - share) <= 2.0 ** -23 * share + 2.0 ** -140, (i, mine)
    assert nears <= max(1, x.shape[0] // 50)
    return tokens


def logits(k, v, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn(k, v, generator=g)
    x.scatter_add_(1, torch.randint(0, v, (k, min(v, 40)), generator=g), 5 + 2 * torch.randn(k, min(v, 40), generator=g))
    return x


SETTINGS = {
    "plain": {}, "cold": dict(t=0.05), "hot": dict(t=30.0), "top-k": dict(top_k=50), "top-1": dict(top_k=1),
    "nucleus": dict(top_p=0.9), "min-p": dict(min_p=0.05), "all": dict(t=0.8, top_k=40, top_p=0.95, min_p=0.02),
    "wide": dict(t=1.5, top_k=5000, top_p=0.999, min_p=1e-6), "greedy": dict(t=0.0), "top-p 0": dict(top_p=0.0),
    "min-p 1": dict(min_p=1.0)}


@pytest.mark.parametrize("name", SETTINGS)
@pytest.mark.parametrize("k,v", [(1, 1), (3, 2), (2, 63), (5, 1000), (2, 1025), (9, 32000), (2, 50257), (3, 128256), (1, 160001), (300, 777)])
def test_settings(name, k, v):
    g = torch.Generator().manual_seed(v)
    u = torch.rand(k, generator=g).tolist()
    check(logits(k, v, v + k), u=u, **{n: [x] * k for n, x in SETTINGS[name].items()})


@pytest.mark.parametrize("v", [100, 32000, 131072])
def test_every_row_its_own(v):
    """Rows of different settings in one call, and rows of a wider buffer."""
    k = 40
    g = torch.Generator().manual_seed(v)
    r = lambda: torch.rand(k, generator=g)
    t = torch.where(r() < 0.2, 0.0, 0.2 + 2 * r()).tolist()
    top_k = torch.where(r() < 0.5, 0.0, torch.exp(11 * r())).int().tolist()
    top_p = torch.where(r() < 0.5, 1.0, r()).tolist()
    min_p = torch.where(r() < 0.5, 0.0, 0.3 * r()).tolist()
    check(logits(k, v + 37, v), vocab=v, t=t, top_k=top_k, top_p=top_p, min_p=min_p, u=r().tolist())


def test_random_numbers_at_their_ends():
    x = logits(8, 3000, 1)
    u = [0.0, -1.0, float("nan"), 1.0, 2.0, float("inf"), 1 - 2.0 ** -24, 2.0 ** -30]
    check(x[:1].repeat(8, 1), u=u)
    check(x[:1].repeat(8, 1), u=u, top_p=[0.7] * 8, top_k=[9] * 8)


def test_settings_that_are_no_limit():
    x, nan = logits(6, 3000, 2), float("nan")
    u = [0.3] * 6
    want = check(x, u=u)
    assert run(x, u=u, t=[1.0] * 6, top_k=[0, -1, 3000, 2 ** 31 - 1, -2 ** 31, 4000], top_p=[1.0, 1.5, nan, 1.0, float("inf"), 1.0],
               min_p=[0.0, -1.0, nan, -float("inf"), 0.0, 0.0])[0] == want


def test_ties():
    """Equal logits go by their ids: all equal, two values, both zeros, more ties than any bin holds."""
    v = 40000
    x = torch.zeros(6, v)
    x[1, ::2] = -0.0
    x[2, ::3] = 1.0
    x[3, 100:] = -1.0
    x[4] = 7.25
    x[5, 39000:] = 3.0
    for settings in [dict(), dict(top_k=[1, 5, 20000, 150, 39999, 1500]), dict(top_p=[0.5, 0.25, 0.9, 0.1, 0.999, 0.3]),
                     dict(top_k=[30000] * 6, top_p=[0.5] * 6), dict(min_p=[0.5] * 6)]:
        check(x, u=[0.1, 0.5, 0.3, 0.77, 0.999, 0.42], **settings)
    # four equal ids: half of the sum is reached by two, exactly
    y = torch.full((2, 500), -float("inf"))
    y[:, [3, 70, 200, 499]] = 1.5
    assert run(y, u=[0.999, 0.5], top_p=[0.5, 1.0])[0] == [70, 200]


@pytest.mark.parametrize("v", [5000, 15000, 36000])
def test_close_logits(v):
    """Thousands of ids within one float32 step of each other's neighbours: every bit of the logit decides."""
    base = np.float32(12.0).view(np.int32)
    bits = base + np.random.default_rng(1).permutation(5000).astype(np.int32)
    x = torch.full((4, v), -100.0)
    x[:, :5000] = torch.from_numpy(bits.view(np.float32).copy())
    check(x, u=[0.1, 0.5, 0.9, 0.3], top_k=[0, 1, 4000, 77], top_p=[1.0, 1.0, 0.5, 1.0])


@pytest.mark.parametrize("v", [2000, 10000, 20000])
def test_masked_and_special_logits(v):
    """-inf and NaN are never chosen, +inf takes everything; rows with nothing left."""
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    x = logits(9, v, 3)
    x[0, 5:] = -inf
    x[1, ::2] = nan
    x[2, [7, 9]] = inf
    x[3] = -inf
    x[4] = nan
    x[5, :v - 1] = low
    x[6] = low
    x[7, 1:] = nan
    x[7, 0] = -inf
    x[8] = torch.where(torch.arange(v) % 2 == 0, 3e38, -3e38)
    for u in (0.0, 0.4, 0.99999):
        tokens = check(x, u=[u] * 9)
        assert tokens[3] == tokens[4] == tokens[7] == -1 and tokens[2] in (7, 9) and tokens[0] < 5
        check(x, u=[u] * 9, top_k=[3] * 9, top_p=[0.9] * 9, min_p=[0.1] * 9)
    greedy = check(x, u=[0.5] * 9, t=[0.0] * 9)
    assert greedy[3] == 0 and greedy[4] == -1 and greedy[7] == 0


@pytest.mark.parametrize("v", [3000, 5000, 12000, 40000])
def test_temperatures_at_their_ends(v):
    x = logits(7, v, 4)
    check(x, u=[0.6] * 7, t=[1e-38, 1e-45, 3e38, float("inf"), -1.0, float("nan"), 1e-3])


def test_frequencies():
    """Evenly spaced u hits every kept id as often as its share says, within one."""
    n, v = 2048, 12
    row = logits(1, v, 5)
    u = [(i + 0.5) / n for i in range(n)]
    tokens, probs = run(row.repeat(n, 1), u=u, top_k=[8] * n)
    w = torch.softmax(row[0].double(), 0)
    w[row[0].argsort(descending=True)[8:]] = 0
    share = w / w.sum()
    count = np.bincount(tokens, minlength=v)
    assert np.all(np.abs(count - n * share.numpy()) <= 1.0)


def test_greedy_is_the_first_tokens_choice():
    """The logits of pp_first_token, sampled at temperature 0, give its tokens."""
    d, v, lengths = 256, 1000, [3, 1, 9, 4]
    cfg = pp.PPConfig(n_layers=1, d_model=d, n_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=1024, vocab=v, dtype=pp.PP_F32,
                      rms_eps=1e-5, rope_theta=1e4)
    dplan = pp.DevicePlan(pp.pp_pack(lengths, 0))
    g = torch.Generator().manual_seed(6)
    hidden, head = torch.randn(sum(lengths), d, generator=g).cuda(), torch.randn(v, d, generator=g).cuda()
    head[500:] = head[:500]                                    # ties
    ws = torch.empty(pp.pp_first_token_workspace_size(cfg, dplan), dtype=torch.uint8, device="cuda")
    tokens, x = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, v, device="cuda")
    pp.pp_first_token(cfg, dplan, hidden, head, ws, tokens, x)
    assert run(x.cpu(), t=[0.0] * 4, u=[0.5] * 4)[0] == tokens.cpu().tolist()


def test_without_prob_and_in_a_graph():
    """prob NULL; recorded once and replayed with new logits, settings and numbers, equal to the eager call."""
    k, v = 6, 32000
    x = logits(k, v, 7).cuda()
    t, tk, tp = torch.full((k,), 0.9, device="cuda"), torch.full((k,), 60, dtype=torch.int32, device="cuda"), torch.full((k,), 0.9, device="cuda")
    u = torch.rand(k, device="cuda")
    ws = torch.empty(max(pp.pp_sample_workspace_size(k, v), 1), dtype=torch.uint8, device="cuda")
    eager, graphed = (torch.empty(k, dtype=torch.int32, device="cuda") for _ in range(2))
    go = lambda out: pp.pp_sample(x, v, k, v, t, tk, tp, None, u, out, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(graphed)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(graphed)
    for i in range(6):
        x.copy_(logits(k, v, 20 + i))
        u.uniform_()
        tk.fill_(1 + 30 * i)
        go(eager)
        torch.cuda.synchronize()
        graph.replay()
        (x + 1).sum()
        torch.cuda.synchronize()
        assert torch.equal(eager, graphed)


def test_two_streams_at_once():
    k, v = 5, 128256
    xs = [logits(k, v, s).cuda() for s in (1, 2)]
    us = [torch.full((k,), 0.37, device="cuda") for _ in range(2)]
    want = [run(x.cpu(), u=[0.37] * k)[0] for x in xs]
    ws = [torch.empty(max(pp.pp_sample_workspace_size(k, v), 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [torch.empty(k, dtype=torch.int32, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for a in range(2):
            pp.pp_sample(xs[a], v, k, v, None, None, None, None, us[a], out[a], ws[a], stream=streams[a])
    torch.cuda.synchronize()
    assert [o.cpu().tolist() for o in out] == want


@pytest.mark.parametrize("k,v", [(1500, 40), (1100, 33000)])
def test_more_rows_than_at_once(k, v):
    """Settings of their own; the larger rows in two sets of launches."""
    g = torch.Generator().manual_seed(5)
    r = lambda n: torch.rand(n, generator=g).tolist()
    check(logits(k, v, 6, 1.5), t=[0.0 if x < 0.1 else 0.3 + 2 * x for x in r(k)], top_k=[int(50 * x) for x in r(k)],
          top_p=[0.3 + x for x in r(k)], min_p=[0.2 * x - 0.05 for x in r(k)], u=r(k))


@pytest.mark.parametrize("v", [1 << 19, (1 << 20) - 1])
def test_largest_vocabularies_of_equal_logits(v):
    """Weights of 2^44 each: sums close to 2^64.  With u and v below 2^24, u v is exact in float64."""
    u = [0.0, 0.25, 0.5, 0.71875, 1 - 2.0 ** -20, 1 - 2.0 ** -24, 1.0, 0.125]
    x = torch.zeros(len(u), v)
    x[2] = 12.0
    x[3] = -float(2 ** 20)
    x[4] = float("inf")
    tokens, prob = run(x, u=u)
    assert tokens == [min(int(a * v), v - 1) for a in u]
    assert all(abs(p * v - 1) <= 2.0 ** -23 for p in prob)
    tokens, prob = run(x, u=u, top_k=[1000] * 8, top_p=[0.5] * 8)
    assert tokens == [min(int(a * 500), 499) for a in u]


# sizes around those where the way changes
WAYS = [(1, 4096), (2, 4097), (3, 8192), (2, 8193), (2, 16384), (2, 16385), (127, 20001), (130, 20001), (128, 32768), (128, 32769)]


@pytest.mark.parametrize("name", ["plain", "hot", "nucleus", "wide", "all", "min-p", "greedy"])
@pytest.mark.parametrize("k,v", WAYS)
def test_ways(name, k, v):
    x = logits(k, v, v + k)
    x[0, 7::5] = float("-inf")
    x[k - 1, 3::9] = float("nan")
    u = torch.rand(k, generator=torch.Generator().manual_seed(k)).tolist()
    check(x, u=u, **{n: [y] * k for n, y in SETTINGS[name].items()})


@pytest.mark.parametrize("k,v", [(2, 4096), (3, 8000), (3, 16384), (128, 32768), (3, 32768)])
def test_ways_with_equal_logits(k, v):
    """More equal logits, and nearly equal ones, than a list holds."""
    x = torch.zeros(k, v)
    x[1] = 1e-6 * torch.randn(v, generator=torch.Generator().manual_seed(2))
    x[k - 1, 5] = float("nan")
    u = [(i + 0.5) / k for i in range(k)]
    check(x, u=u)
    check(x, u=u, top_k=[v // 3] * k, top_p=[0.75] * k)
    tokens, prob = run(x, u=u, t=[1e-30] * k)            # exponents of 2^30 and more
    for i in range(k):
        token, share, near = definition(x[i].numpy(), 1e-30, u=u[i])
        assert near or (tokens[i] == token and abs(prob[i] - share) <= 2.0 ** -23 * share)
