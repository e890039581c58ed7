"""Infinities in V of packed prompts over pages: the sign that they have in the outputs of bf16 models.

An output is the pair hi = bf16(x), lo = bf16(x - hi), so that of an infinity hi alone tells its sign (lo is NaN).  A token that sees
some slots of a 32-slot block and not others has its infinities counted apart from the products, by marks, and is infinite with their
sign.  Where all rows of a matrix product see the block, weights meet the infinity plane by plane: a plane of 0 makes that NaN, which
the definition allows; finite, or of the other sign, it is never.

Marked ``gpu``: needs an MI355X and ``libham.so`` built in-tree.
"""
import pytest
import torch

from synth.configs import BF16
from tests.gpu_util import act_rows
from tests.paged_planes import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


@pytest.fixture(scope="module")
def ham():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2505_20438_amd import ham
    ham.load_library()
    return ham


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# tiles of few and of many slots, the long prompts' kernel with two key shares, split and not, one share of 4 and of 8 waves
@pytest.mark.parametrize("H,Hk,hd,P,rows", [
    (8, 2, 128, 16, [(0, 200), (50, 70)]), (4, 4, 64, 32, [(300, 90), (0, 33)]), (16, 1, 128, 32, [(0, 20), (64, 40)]), (8, 2, 64, 32, [(3000, 60)]),
    (32, 8, 64, 32, [(300, 1100), (0, 33)]), (32, 8, 128, 16, [(0, 1500)]), (16, 1, 64, 16, [(17001, 260)]), (16, 1, 128, 32, [(30, 2150), (0, 20)]),
    (32, 8, 128, 32, [(0, 300)] * 20), (32, 8, 64, 64, [(40, 350)] * 18), (16, 8, 128, 32, [(0, 7000)]), (16, 8, 64, 64, [(8000, 2100), (0, 900)])])
@pytest.mark.parametrize("bad", [INF, -INF])
def test_the_sign_of_an_infinity_in_v(ham, H, Hk, hd, P, rows, bad):
    offsets, lens = [0], [a + b for a, b in rows]
    for _, c in rows:
        offsets.append(offsets[-1] + c)
    s, pool, g = make(ham, BF16, H, Hk, hd, P, lens)
    held, c = rows[0]
    at = held + c // 2 + 3                  # a slot in the middle of the first row's tokens
    k, v = (x[:, at].clone() for x in pool.keys_values(0, at + 1))
    v[0, 5] = bad
    pool.append(0, at, k[None], v[None])
    q = act_rows(torch, torch.randn(offsets[-1], H * hd, generator=g), BF16).to(DEV)
    out, err = torch.zeros_like(q), i32([0] * s.rows)
    ws = torch.full((ham.ham_op_paged_workspace_bytes(s),), 0x5A, dtype=torch.uint8, device=DEV)
    ham.ham_op_paged_prompt(s, q, i32(offsets), pool.data.to(DEV), i32(pool.table), i32(lens), max(lens), out, err, ws,
                            torch.cuda.current_stream().cuda_stream)
    assert err.tolist() == [0] * s.rows
    hi, lo = out.cpu().float().view(-1, 2, H, hd).unbind(1)
    first, seen = at - held, range(at - held, c)   # packed rows of the first row that see the slot
    x = hi[first:c, :H // Hk, 5]
    assert torch.all((x == bad) | torch.isnan(x))
    # tokens at slots of the same block that do not see all of it
    part = [i for i in seen if held + i + 1 < at // 32 * 32 + 32]
    assert len(part) > 0 and torch.all(hi[part][:, :H // Hk, 5] == bad)
    whole = torch.ones(hi.shape, dtype=torch.bool)
    whole[first:c, :H // Hk, 5] = False
    assert torch.isfinite(hi[whole]).all() and torch.isfinite(lo[whole]).all()
