"""No bf16 plane of the weights is lost in the attention over pages: every kernel and form of it, on inputs (``paged_planes``) that a
lost plane shows in, at few slots and at more than 16,384.

Marked ``gpu``: needs an MI355X and ``libham.so`` built in-tree.
"""
import pytest
import torch

from tests import paged_planes as pp
from tests.gpu_util import act_rows, from_act

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ham():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2505_20438_amd import ham
    ham.load_library()
    return ham


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def hold(out, q, pool, seen, at, H, hd, dtype):
    n = len(at)
    got, qd = (from_act(torch, x[at], H * hd, dtype).double().view(n, H, hd) for x in (out.cpu(), q))
    assert pp.errors(got, *pp.attention(pool, qd, seen), dtype).max() < 1.0


def setup(ham, dtype, H, hd, pool, s, g, n):
    q = act_rows(torch, pp.SIGMA_Q * torch.randn(n, H * hd, generator=g), dtype)
    ws = torch.full((ham.ham_op_paged_workspace_bytes(s),), 0x5A, dtype=torch.uint8, device=DEV)
    return q, torch.zeros_like(q, device=DEV), i32([0] * s.rows), ws, torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype,H,Hk,hd,P,lens", pp.ATTENTION)
def test_of_one_token(ham, dtype, H, Hk, hd, P, lens):
    s, pool, g = pp.make(ham, dtype, H, Hk, hd, P, lens)
    q, out, err, ws, st = setup(ham, dtype, H, hd, pool, s, g, len(lens))
    ham.ham_op_paged_attention(s, q.to(DEV), pool.data.to(DEV), i32(pool.table), i32(lens), i32([1] * s.rows), max(lens), out, err, ws, st)
    assert err.tolist() == [0] * s.rows
    hold(out, q, pool, list(enumerate(lens)), list(range(len(lens))), H, hd, dtype)


@pytest.mark.parametrize("dtype,H,Hk,hd,P,rows,kernel", pp.PROMPTS)
def test_of_a_prompt(ham, dtype, H, Hk, hd, P, rows, kernel):
    lens, offsets = [a + b for a, b in rows], [0]
    for _, c in rows:
        offsets.append(offsets[-1] + c)
    s, pool, g = pp.make(ham, dtype, H, Hk, hd, P, lens)
    q, out, err, ws, st = setup(ham, dtype, H, hd, pool, s, g, offsets[-1])
    ham.ham_op_paged_prompt(s, q.to(DEV), i32(offsets), pool.data.to(DEV), i32(pool.table), i32(lens), max(lens), out, err, ws, st)
    assert err.tolist() == [0] * s.rows
    tokens = pp.some_tokens(rows)
    hold(out, q, pool, [(r, n) for _, r, n in tokens], [i for i, _, _ in tokens], H, hd, dtype)
