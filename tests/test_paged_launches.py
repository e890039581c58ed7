"""What a call on a paged KV cache may hold at most, without a GPU: append's launches (``csrc/launch_rules.h``), and the refusals past
the limits that include/ham_ops.h names.

Every call here is refused before anything is launched; pointers are numbers that nothing reads.
"""
import ctypes
import os
import subprocess
import tempfile

import pytest

from paper_2505_20438_amd import ham
from synth.configs import BF16

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_20438_amd", "csrc")


@pytest.fixture(scope="module")
def rules():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "r.cpp"), os.path.join(d, "r.so")
        with open(src, "w") as f:
            f.write('#include "launch_rules.h"\nextern "C" {\n'
                    'long long steps(long long N, long long R) { return ham::paged_append_steps(N, R); }\n'
                    'int groups(int N, int R, int heads) { return ham::paged_append_groups(N, R, heads); }\n'
                    'long long workgroups(int N, int R, int heads) { return ham::paged_append_workgroups(N, R, heads); }\n'
                    'int fits(long long N, int Hk) { return ham::paged_append_fits(N, Hk); }\n}\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        r = ctypes.CDLL(out)
        r.steps.argtypes, r.steps.restype, r.workgroups.restype = [ctypes.c_longlong] * 2, ctypes.c_longlong, ctypes.c_longlong
        r.fits.argtypes = [ctypes.c_longlong, ctypes.c_int]
        yield r


def test_what_append_takes_fits_a_launch(rules):
    for Hk in (1, 2, 3, 8, 32, 127, 512, 1024):
        most = (1 << 27) // Hk
        for N in (1, 2, 63, 64, 65, 4095, 4096, 4097, 100000, 1 << 20, most - 1, most):
            N = min(N, most, 1 << 24)
            assert rules.fits(N, Hk)
            for R in (1, 2, 63, 64, 65, 1000, 4096):
                for heads in (Hk, 2 * Hk):
                    n = rules.workgroups(N, R, heads)
                    assert rules.steps(N, R) * rules.groups(N, R, heads) <= n < 1 << 24
        assert most >= 1 << 24 or not rules.fits(most + 1, Hk)
    assert rules.fits(4096, 1024)     # a token of each of 4,096 rows, 1,024 kv heads


def call(name, s, args):
    lib = ham.load_library()
    rc = getattr(lib, "ham_op_paged_" + name)(ctypes.byref(s), *args, None)
    return rc, lib.ham_last_error()


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ham.LIB_PATH):
        pytest.skip("libham.so not built")


BIG = 1 << 60


@pytest.mark.parametrize("N,Hk", [((1 << 17) + 1, 1024), (1 << 24, 9), ((1 << 22) + 1, 32)])
def test_append_past_its_limit_is_refused(N, Hk):
    for rows in (1, 4096):
        rc, why = call("append", ham.paged_shape(BF16, rows, Hk, Hk, 64, 256, 9, 1 << 16), [N] + [256] * 7 + [BIG, 256, 256])
        assert rc == ham.HAM_EINVAL and b"too large" in why


@pytest.mark.parametrize("N,rows,H,Hk", [((1 << 16) + 1, 1, 1024, 1024), ((1 << 22) + 1, 1, 16, 1), (1 << 24, 1, 5, 1), (8192, 4096, 1024, 1024)])
def test_prompts_past_their_limit_are_refused(N, rows, H, Hk):
    assert Hk * min(N, (N * (H // Hk) + 15 * rows) // 16) > 1 << 22
    rc, why = call("prompt", ham.paged_shape(BF16, rows, H, Hk, 64, 256, 9, 1 << 16), [N, 256, 256, 256, BIG, 256, 256, 4000, 256, 256, 256, BIG])
    assert rc == ham.HAM_EINVAL and b"too large" in why
