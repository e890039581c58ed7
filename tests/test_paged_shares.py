"""The shares that the attention of one token over pages cuts its rows into (``paged_share_size`` of ``csrc/launch_rules.h``), up to
the longest rows that a shape may have."""
import ctypes
import os
import random
import subprocess
import tempfile

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_20438_amd", "csrc")


@pytest.fixture(scope="module")
def rules():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "r.cpp"), os.path.join(d, "r.so")
        with open(src, "w") as f:
            f.write('#include "launch_rules.h"\nextern "C" {\n'
                    'int size(long long all, int most, int R, int shares) { return ham::paged_share_size(all, most, R, shares); }\n'
                    'int shares_of(int R, int Hk) { return ham::paged_attn_shares(R, Hk); }\n}\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        r = ctypes.CDLL(out)
        r.size.argtypes = [ctypes.c_longlong] + [ctypes.c_int] * 3
        yield r


def check(rules, blocks, Hk):
    R, n = len(blocks), rules.shares_of(len(blocks), Hk)
    size = rules.size(sum(blocks), max(blocks), R, n)
    want = max(-(-sum(blocks) // (n - min(R, n // 2))), 8, -(-max(blocks) // 64))
    assert size == want or (sum(blocks) == 1 << 32 and size in (want, want - 1))
    cut = [max(1, -(-b // size)) for b in blocks]
    assert sum(cut) <= n + R and max(cut) <= 64


@pytest.mark.parametrize("blocks", [1 << 20, 1 << 19])     # 2^24 slots, of fp32 and of bf16
def test_rows_of_2_24_slots(rules, blocks):
    for R in (1, 2, 64, 65, 2047, 2048, 2049, 4095, 4096):
        for Hk in (1, 2, 3, 4):
            if R * Hk <= 16384:
                check(rules, [blocks] * R, Hk)
                check(rules, [blocks] * (R - 1) + [1], Hk)


def test_ragged_rows(rules):
    g = random.Random(6)
    for _ in range(2000):
        R = g.choice((1, 3, 64, 100, 2500, 4096))
        top = g.choice((9, 300, 1 << 14, 1 << 20))
        check(rules, [g.choice((0, 1, g.randint(0, top), top)) for _ in range(R)], g.choice((1, 2, 4)))
