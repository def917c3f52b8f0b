"""pp_sample on rows whose ids reach far below the likeliest one: a confident logit over a bulk, cold temperatures, every
limit, and random numbers up to the end.  Rows that one workgroup reads and rows in parts are held to the same definition.

Weights are counted in units of 2^(E - 44), E the whole number at or above the likeliest id's logit in powers of two.  A sum
of n ids' weights is off by half a unit for each of them (an id's own rounding), where the row is in parts by half a unit for
each of 16 parts' 1440 bins, and by 2^-52 of itself; a bound (a float32 number times a sum) as its sum is."""
import itertools

import numpy as np
import pytest
import torch

from .gpu_util import require_gpu
from .test_gpu_sample import run

pytestmark = pytest.mark.gpu

LOG2E = 1.4426950408889634


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Row:
    """A row's ids in order with their weights in units."""

    def __init__(self, x, t):
        x = x.astype(np.float64)
        ids = np.flatnonzero(x > -np.inf)
        self.order = ids[np.argsort(-x[ids], kind="stable")]
        y = x[self.order]
        c = LOG2E / np.float64(np.float32(t))
        depth = np.ceil(y[0] * c) - y * c
        # ids of half a unit and more; of the last of these, up to a 128th of an octave above it, any number may be none
        self.n, self.sure = (int((depth < 45 + e).sum()) for e in (2.0 ** -30, -2.0 ** -7 - 2.0 ** -30))
        self.w = np.exp2(44 - depth[:self.n])
        self.cum = np.cumsum(np.rint(self.w))
        self.share = np.exp((y[:self.n] - y[0]) / np.float64(np.float32(t)))
        self.slack = 0.5 * self.n + 0.5 * 16 * 1440 + 2.0 ** -50 * self.cum[-1]

    def check(self, token, prob, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
        cum, place = self.cum, np.flatnonzero(self.order[:self.n] == token)
        assert place.size == 1, "an id that is never chosen"
        j = int(place[0])
        # how many are kept, at least and at most
        lo, hi = (min(n, top_k) if top_k > 0 else n for n in (self.sure, self.n))
        if top_p < 1:
            p = float(np.float32(top_p))
            reach = np.searchsorted(cum[:hi], [max(p * cum[lo - 1] - self.slack, 1.0), p * cum[hi - 1] + self.slack]) + 1
            lo, hi = min(int(reach[0]), lo), min(int(reach[1]), hi)
        if min_p > 0:
            m = float(np.float32(min_p))
            lo, hi = min(lo, int((self.share >= m * (1 + 2.0 ** -50)).sum())), min(hi, int((self.share >= m * (1 - 2.0 ** -50)).sum()))
        assert 0 < lo <= hi
        if u >= 1:
            assert lo - 1 <= j <= hi - 1, "not the last kept id"
        else:
            u = float(np.float32(u))
            assert j < hi, "an id that is not kept"
            assert cum[j] > u * cum[lo - 1] - self.slack, "an id before the place"
            assert j == 0 or cum[j - 1] <= u * cum[hi - 1] + self.slack, "an id behind the place"
        most, least = self.w[j] / (cum[lo - 1] - self.slack), self.w[j] / (cum[hi - 1] + self.slack)
        assert least * (1 - 2.0 ** -23) - 2.0 ** -140 <= prob <= most * (1 + 2.0 ** -23) + 2.0 ** -140


def confident(rows, v, seed, winner):
    """A bulk of standard deviation 2.5 and one id (rows take turns in `winner`) above it."""
    g = torch.Generator().manual_seed(seed)
    x = 2.5 * torch.randn(rows, v, generator=g)
    at = torch.randint(0, v, (rows,), generator=g)
    for i in range(rows):
        x[i, at[i]] = winner[i % len(winner)]
    return x


def check(x, rows_of_a_call, **settings):
    for a in range(0, x.shape[0], rows_of_a_call):
        part = {n: s[a:a + rows_of_a_call] for n, s in settings.items()}
        tokens, probs = run(x[a:a + rows_of_a_call], **part)
        for i, (token, prob) in enumerate(zip(tokens, probs)):
            mine = {n: s[i] for n, s in part.items()}
            try:
                Row(x[a + i].numpy(), mine.pop("t")).check(token, prob, **mine)
            except AssertionError as e:
                raise AssertionError(f"row {a + i}, {settings['t'][a + i]}, {mine}: {token}, share {prob}: {e}") from None


WINNERS = [10.0, 12.0, 16.0, 20.0, 23.0, 27.0, 31.0, 39.0, 49.0]
TEMPERATURES = [0.2, 0.25, 0.3, 0.4, 0.5, 0.6, 0.8, 1.0]
LIMITS = {"top-k": {}, "top-k and top-p": dict(top_p=0.9), "all": dict(top_p=0.999, min_p=1e-9), "min-p": dict(min_p=1e-12)}


@pytest.mark.parametrize("limits", LIMITS)
@pytest.mark.parametrize("v,rows_of_a_call", [(2000, 72), (16384, 72), (32000, 1), (32000, 24), (50257, 24), (128256, 72)])
def test_confident_rows(v, rows_of_a_call, limits):
    rows = 24 if rows_of_a_call == 1 else 72
    pairs = list(itertools.product(WINNERS, TEMPERATURES))[::72 // rows]
    x = confident(rows, v, v + rows, [w for w, _ in pairs])
    g = torch.Generator().manual_seed(rows)
    k = [[50, 2, 200, 1, 1000][i % 5] for i in range(rows)]
    u = [[0.0, 0.5, 0.9, 1 - 2.0 ** -24, float(torch.rand(1, generator=g))][i // 2 % 5] for i in range(rows)]
    check(x, rows_of_a_call, t=[t for _, t in pairs], u=u, **({} if limits == "min-p" else dict(top_k=k)),
          **{n: [y] * rows for n, y in LIMITS[limits].items()})


@pytest.mark.parametrize("v", [800_000, 2 ** 20 - 1])
def test_groups_of_equal_logits_in_the_largest_rows(v):
    """Sums close to 2^64, and an id that lies among equal ones behind others."""
    g = torch.Generator().manual_seed(v)
    mixed = torch.randperm(v, generator=g)
    x = torch.zeros(8, v)
    x[0:3, mixed[:v // 4]] = -1e-7
    x[3, mixed[:v // 2]] = -0.25
    x[4, mixed[:v // 100]] = -1e-7
    x[5, mixed[:v - v // 100]] = -3e-7
    x[6:] = -10 - torch.randn(2, v, generator=g)
    x[7] = torch.round(4 * x[7]) / 4                         # some dozens of values
    t = [1.0] * 6 + [1e6] * 2
    u = [0.9, 0.76, 1 - 2.0 ** -24, 0.8, 0.995, 0.5, 0.97, 0.9]
    check(x, 8, t=t, u=u)
    check(x, 8, t=t, u=u, top_k=[v - 5] * 8, top_p=[0.95] * 8)


@pytest.mark.parametrize("limits", ["none", *LIMITS])
@pytest.mark.parametrize("v,rows_of_a_call", [(2000, 36), (16384, 36), (32000, 1), (32000, 36), (128256, 36), (128256, 1)])
def test_last_kept_id(v, rows_of_a_call, limits):
    """u of 1 and more."""
    rows = 6 if rows_of_a_call == 1 else 36
    pairs = list(itertools.product(WINNERS, TEMPERATURES))[1::72 // rows]
    x = confident(rows, v, v + rows + 1, [w for w, _ in pairs])
    k = [[50, 2, 200, 1, 1000][i % 5] for i in range(rows)]
    check(x, rows_of_a_call, t=[t for _, t in pairs], u=[[1.0, 2.0, float("inf")][i % 3] for i in range(rows)],
          **({} if limits in ("none", "min-p") else dict(top_k=k)), **{n: [y] * rows for n, y in LIMITS.get(limits, {}).items()})


@pytest.mark.parametrize("v", [4000, 16000, 40000])
def test_last_kept_id_of_many_likely_ones(v):
    """Sums past 2^53, whose last ids are a unit or two each; in lists, and by descent (more than 4096 equal ids)."""
    x = torch.full((6, v), -float("inf"))
    for i, n in enumerate([1000, 1500, 2000, 3000, v // 2, 3 * v // 4]):
        x[i, :n] = 0.0
        x[i, n:n + 600] = -30.0 - 0.25 * (torch.arange(600) % 3)        # 1.6, 1.3 and 1.0 units
    u = [1.0] * 6
    check(x, 6, t=[1.0] * 6, u=u)
    check(x, 6, t=[1.0] * 6, u=u, top_k=[1100, 1601, 2555, 100, v // 2 + 599, 3 * v // 4 + 250])
    check(x, 6, t=[1.0] * 6, u=u, min_p=[9e-14, 7.5e-14, 0.5, 9e-14, 9e-14, 7.5e-14])
