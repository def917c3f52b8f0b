"""The choice between the 8-bit GEMM's kernels, asked on the CPU (``tests/host/quant_choice.cpp``): the sizes of
the GPU tests reach every way a call can go, so that new constants of the estimate leave none untested."""
import math
import os
import random
import shutil
import subprocess

import pytest

from . import test_gpu_quant_ways as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2404_09529_amd", "csrc")
LARGE = {2: "192x192", 3: "192x256", 4: "256x256"}
TILES = ["32x64", "64x64", "64x128", "128x128", "128x256"]


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("choice") / "quant_choice")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "quant_choice.cpp"), "-o", exe], check=True, timeout=300)

    def ask(calls):
        r = subprocess.run([exe], input="\n".join("%d %d %d %d" % c for c in calls), capture_output=True, text=True,
                           check=True, timeout=300)
        return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]

    return ask


def way(call, choice):
    """As the keys of ROWS (no list: entries -1) and of LISTS."""
    M, N, K, entries = call
    kind, tile, shares, big = choice
    full = () if entries < 0 else (entries == -(-M // 256),)
    if kind == 0:
        return ("few", tile, 1 if M <= 16 else 2 if M <= 32 else 4) + full
    if kind == 1:
        return ("tile", TILES[tile], shares, big > 0) + full
    return (LARGE[kind],) + full


def test_sizes_go_the_ways_they_are_named_for(choose):
    calls = [(*size, -1) for size in W.ROWS.values()]
    for rows, capacity, length, N, K in W.LISTS.values():
        calls.append((rows * capacity, N, K, W.list_plan(rows, capacity, length).n_mtiles))
    assert [way(c, r) for c, r in zip(calls, choose(calls))] == [*W.ROWS, *W.LISTS]


def test_no_other_way_is_common(choose):
    """Of 200,000 sizes (a list has more than one tile) no other way is taken by more than a few."""
    rng = random.Random(3)

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    calls = []
    for i in range(200000):
        M = log(257, 40000) if i % 2 else log(1, 40000)
        full = -(-M // 256)
        entries = -1 if i % 2 == 0 else full if i % 4 == 1 else rng.randint(1, full)
        calls.append((M, 16 * log(1, 2000), 16 * log(1, 1200), entries))
    seen = {}
    for c, r in zip(calls, choose(calls)):
        w = way(c, r)
        seen[w] = seen.get(w, 0) + 1
    assert {w for w, n in seen.items() if n >= 10} <= {*W.ROWS, *W.LISTS}


def test_few_rows_fit_a_launch(choose):
    """A launch holds fewer than 2^32 threads: the kernel for few rows takes no columns past that."""
    rng = random.Random(4)
    calls = [(M, N, K, -1) for M in (1, 16, 17, 32, 33, 64) for K in (16, 64, 128, 1024, 131056)
             for N in (2 ** 27, 2 ** 28 - 32, 2 ** 28, 2 ** 29, 2 ** 30 - 64, 2 ** 30, 2 ** 31 - 512)]
    calls += [(rng.randint(1, 64), 16 * rng.randint(2 ** 22, 2 ** 27 - 32), 16 * int(2 ** rng.uniform(0, 8)), -1)
              for _ in range(20000)]
    few = 0
    for (M, N, K, _), (kind, blocks, _, _) in zip(calls, choose(calls)):
        if kind == 0:
            few += 1
            assert -(-N // (16 * blocks)) * (256 if blocks == 4 else 512) < 2 ** 32, (M, N, K)
    assert few > 0
