"""The operators on a paged KV cache at the largest sizes that a shape may have.

Marked ``gpu``: needs an MI355X and ``libham.so`` built in-tree.
"""
import pytest
import torch

from synth.configs import BF16, F32
from tests.paged_ref import places

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ham():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2505_20438_amd import ham
    ham.load_library()
    return ham


def test_attention_of_rows_with_2_31_blocks_together(ham):
    """2,060 rows of 2^24 slots, all of them in three pages: 2^31 blocks of 16.  Keys are 0, so that all weights are 1, and values -1, 0
    and 1: sums of up to 2^24 of them are exact in fp32 in any order, and the division by their number and the factors of the join
    round, three times by 2^-24 at most."""
    R, P, top = 2060, 256, 1 << 24
    entries = top // P
    s = ham.paged_shape(F32, R, 1, 1, 64, P, 3, entries)
    g = torch.Generator().manual_seed(2)
    v = torch.randint(-1, 2, (3, P, 64), generator=g)
    pool = torch.zeros(3, 1, 2, P * 64)
    pool[:, 0, 1] = v.view(3, P // 4, 4, 64).transpose(2, 3).reshape(3, P * 64).float()
    lens = [top - (0 if r < 2050 else 777 * r) for r in range(R)]
    assert sum(-(-n // 16) for n in lens) >= 1 << 31
    r, e = torch.arange(R, device=DEV, dtype=torch.int32)[:, None], torch.arange(entries, device=DEV, dtype=torch.int32)
    table = (r + e * (1 + r % 2)) % 3
    q, n = torch.randn(R, 64, generator=g).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, err = torch.full((R, 64), 7.0, device=DEV), torch.zeros(R, dtype=torch.int32, device=DEV)
    ws = torch.full((ham.ham_op_paged_workspace_bytes(s),), 0x5A, dtype=torch.uint8, device=DEV)
    ham.ham_op_paged_attention(s, q, pool.to(DEV), table, n, torch.ones_like(n), top, out, err, ws, torch.cuda.current_stream().cuda_stream)
    page, part = v.sum(1), v.cumsum(1)
    want = torch.zeros(R, 64, dtype=torch.float64)
    for i, slots in enumerate(lens):
        whole, rest = divmod(slots, P)
        ids = (i + torch.arange(whole + 1) * (1 + i % 2)) % 3
        total = (torch.bincount(ids[:whole], minlength=3)[:, None] * page).sum(0)
        if rest:
            total = total + part[ids[whole], rest - 1]
        want[i] = total.double() / slots
    assert err.tolist() == [0] * R
    assert torch.all((out.cpu().double() - want).abs() <= 2.0 ** -22 * want.abs())


def test_append_of_a_token_of_4096_rows_with_1024_kv_heads(ham):
    """Row r's token goes to slot r % 16 of page r // 16.  Angles are 0: rotated rows are the rows themselves, rounded."""
    R, H, hd, P = 4096, 1024, 64, 16
    s = ham.paged_shape(BF16, R, H, H, hd, P, R // P, 1)
    g = torch.Generator(device=DEV).manual_seed(3)
    qkv = torch.randn(R, 3, H, hd, generator=g, device=DEV)
    one, r = torch.ones(R, hd // 2, device=DEV), torch.arange(R + 1, dtype=torch.int32, device=DEV)
    pool = torch.full((R // P, H, 2, P * hd), float("nan"), dtype=torch.bfloat16, device=DEV)
    q, err = torch.zeros(R, 2 * H * hd, dtype=torch.bfloat16, device=DEV), torch.zeros(R, dtype=torch.int32, device=DEV)
    ham.ham_op_paged_append(s, qkv.view(R, -1), one, torch.zeros_like(one), r, r[:R] % P, (r[:R] // P).view(R, 1), pool, q, err,
                            torch.cuda.current_stream().cuda_stream)
    assert int(err.abs().max()) == 0
    k_at, v_at = (t.to(DEV) for t in places(P, hd, 8))
    kv = qkv[:, 1:].bfloat16().view(R // P, P, 2, H, hd)
    for j, at in ((0, k_at), (1, v_at)):
        got = pool[:, :, j][:, :, at].permute(0, 2, 1, 3)          # [page][slot][kv head][channel]
        assert torch.equal(got, kv[:, :, j])
    hi = qkv[:, 0].reshape(R, -1).bfloat16()
    assert torch.equal(q, torch.cat([hi, (qkv[:, 0].reshape(R, -1) - hi.float()).bfloat16()], 1))
