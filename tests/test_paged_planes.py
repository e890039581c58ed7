"""The cases of paged_planes.py: the attention with every bf16 plane of the weights stays well below its bound, one with a plane less
exceeds it for every token that sees many slots, all in pairs, and every head; and each case is in the kernel that it says.

One kv head and at most two q-heads of a case are looked at here: the others' are of the same distribution.
"""
import ctypes
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2505_20438_amd import ham
from synth.configs import BF16
from tests import paged_planes as pp
from tests.gpu_util import act_rows, from_act

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_20438_amd", "csrc")


def hold(dtype, H, hd, pool, g, seen):
    n = len(seen)
    q = from_act(torch, act_rows(torch, pp.SIGMA_Q * torch.randn(n, H * hd, generator=g), dtype), H * hd, dtype).double().view(n, H, hd)
    want, spread = pp.attention(pool, q, seen)

    def part(*planes):
        return pp.errors(pp.attention(pool, q, seen, planes)[0], want, spread, dtype)
    many = torch.tensor([x >= pp.MANY and x % 2 == 0 for _, x in seen])
    assert many.any()
    if dtype != BF16:
        assert float(part(0, "").max()) <= 0.5
        return
    assert float(part(3, "cut").max()) <= 0.5
    assert float(part(2, "cut")[many].min()) >= 1.5 and float(part(2, "near")[many].min()) > 1.0


@pytest.mark.parametrize("dtype,H,Hk,hd,P,lens", pp.ATTENTION)
def test_a_lost_plane_of_one_token_shows(dtype, H, Hk, hd, P, lens):
    H = min(2, H // Hk)
    s, pool, g = pp.make(ham, dtype, H, 1, hd, P, lens)
    hold(dtype, H, hd, pool, g, list(enumerate(lens)))


@pytest.mark.parametrize("dtype,H,Hk,hd,P,rows,kernel", pp.PROMPTS)
def test_a_lost_plane_of_a_prompt_shows(dtype, H, Hk, hd, P, rows, kernel):
    H, rows = min(2, H // Hk), rows[-2:]
    s, pool, g = pp.make(ham, dtype, H, 1, hd, P, [a + b for a, b in rows])
    hold(dtype, H, hd, pool, g, [(r, n) for _, r, n in pp.some_tokens(rows)])


def test_each_case_is_in_its_kernel():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "r.cpp"), os.path.join(d, "r.so")
        with open(src, "w") as f:
            f.write('#include "launch_rules.h"\nextern "C" {\n'
                    'int as_tiles(int N, int R, int Hk, int grp, int kv) { return ham::paged_prompt_tiles(N, R, Hk, grp, kv); }\n'
                    'int shares(int N, int R, int Hk, int grp, int kv) { return ham::paged_prompt_grid(N, R, Hk, grp, kv).shares; }\n'
                    'int waves(int N, int Hk, int grp, int hd, int kv) { return ham::paged_prompt_waves(N, Hk, grp, hd, kv); }\n}\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
        r = ctypes.CDLL(out)
    forms = set()
    for dtype, H, Hk, hd, P, rows, kernel in pp.PROMPTS:
        N, kv, grp = sum(c for _, c in rows), max(a + c for a, c in rows), H // Hk
        got = 0
        if dtype == BF16 and not r.as_tiles(N, len(rows), Hk, grp, kv):
            ks = r.shares(N, len(rows), Hk, grp, kv)
            got = (ks, 8 if ks == 2 else r.waves(N, Hk, grp, hd, kv))
            forms.add((hd, *got))
        assert got == kernel, (rows, got)
    assert forms == {(hd, *k) for hd in (64, 128) for k in ((2, 8), (1, 8), (1, 4))}
