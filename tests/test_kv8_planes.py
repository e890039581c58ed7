"""The bounds of kv8_planes.py: the attention with every bf16 plane stays well below them, one with a plane less exceeds them for
every row and head."""
import os

import pytest
import torch

from paper_2505_20438_amd import ham
from synth.configs import BF16, F32
from tests import kv8_planes

SHAPES = [(BF16, 4, 1, 64, [300, 1001]), (BF16, 16, 1, 128, [2100, 220]), (F32, 4, 2, 64, [300, 1000]), (F32, 9, 3, 128, [2100, 220])]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(ham.LIB_PATH):
        pytest.skip("libham.so not built")


@pytest.mark.parametrize("dtype,H,Hk,hd,lens", SHAPES)
def test_bounds_tell_a_lost_plane(dtype, H, Hk, hd, lens):
    for pairs in (True, False):
        _, ref, _, q = kv8_planes.inputs(ham, dtype, H, Hk, hd, lens, pairs)
        out, spread = kv8_planes.expected(ref, q, lens)

        def part(**kw):
            return kv8_planes.errors(kv8_planes.emulated(ref, q, lens, dtype, **kw), out, spread, dtype)
        assert float(part().max()) <= 0.5
        if pairs:
            assert float(part(p_planes=2).min()) >= 1.5
        elif dtype == F32:
            assert float(part(p_planes=2).min()) >= 1.5 and float(part(q_planes=2).min()) > 1.0
        assert float(part(q_planes=1).min()) >= 1.5


def test_inputs_with_pairs_cancel():
    lens = [300, 1001]
    _, ref, _, q = kv8_planes.inputs(ham, BF16, 4, 1, 64, lens, True)
    out, spread = kv8_planes.expected(ref, q, lens)
    assert float((out.norm(dim=-1) / spread.norm(dim=-1)).max()) <= 0.05
    assert torch.allclose(out, ref.attention(q, lens), rtol=0, atol=1e-14)
