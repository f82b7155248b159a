"""The mask's index arithmetic over the whole range of sizes that the attention calls take (up to 2^30 tokens), against integers of any
size.  Compiled for the host: no GPU."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 1 << 30


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("mask") / "check")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", exe,
                    os.path.join(HERE, "attention_mask_check.cu")], check=True)

    def run(cases):
        lines = "".join(" ".join(str(v) for v in c) + "\n" for c in cases)
        out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return run


def _want(q_len, k_len, causal, window, keys, i, j):
    """Ranges that select the same pairs as the definition: empty where it has none, else equal."""
    d = k_len - q_len
    lo, hi = (max(0, i + d - window) if window >= 0 else 0), (min(keys, i + d + 1) if causal else keys)
    qlo, qhi = (max(0, j - d) if causal else 0), (min(q_len, j - d + window + 1) if window >= 0 else q_len)
    return lo, hi, qlo, qhi


def test_ranges_over_all_sizes(check):
    rng = random.Random(3)
    size = lambda: rng.choice([1, rng.randint(1, 300), rng.randint(1, MOST), MOST - rng.randint(0, 3), MOST])
    cases = [(MOST, 1, 0, MOST, 1, 0, 0), (MOST, 1, 1, 1 << 40, 1, MOST - 1, 0), (MOST, MOST, 0, MOST - 2, MOST, MOST - 1, MOST - 1)]
    for _ in range(20000):
        q_len, k_len = size(), size()
        window = rng.choice([-1, 0, rng.randint(0, 300), rng.randint(0, k_len), max(0, k_len - rng.randint(0, 3)), rng.randint(0, 1 << 62)])
        keys = rng.choice([k_len, rng.randint(1, k_len)])
        cases.append((q_len, k_len, rng.randint(0, 1), window, keys, rng.choice([0, q_len - 1, rng.randrange(q_len)]), rng.choice([0, keys - 1, rng.randrange(keys)])))
    got = check(cases)
    assert len(got) == len(cases)
    for c, g in zip(cases, got):
        q_len, k_len, causal, window, keys, i, j = c
        lo, hi, qlo, qhi = _want(*c)
        assert (g[0], g[1]) == (lo, hi) or (lo >= hi and g[0] >= g[1]), (c, g)
        assert (g[2], g[3]) == (qlo, qhi) or (qlo >= qhi and g[2] >= g[3]), (c, g)
        # keys in front of the first, queries in front of the first and from the end on: exactly those that see nothing, where the others may
        assert g[4] == (max(0, k_len - q_len - window) if window >= 0 else 0)
        assert g[5] == (max(0, q_len - k_len) if causal else 0)
        end = min(q_len, keys - k_len + q_len + window) if window >= 0 else q_len
        assert g[6] == end and ((i < g[5] or i >= g[6]) == (lo >= hi)), (c, g)
