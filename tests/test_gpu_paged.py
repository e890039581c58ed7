"""The operators on a paged KV cache (``ham_op_paged_*``) against their definition (``paged_ref``; tolerances there), through
the C ABI.

Marked ``gpu``: needs an MI355X and ``libham.so`` built in-tree.
"""
import random

import pytest
import torch

from synth.configs import BF16, F32
from tests import kv8_planes
from tests.attention_bounds import FILLED_TOL
from tests.gpu_util import act_rows, from_act
from tests.kv8_ref import act64, rope64, storage, stored
from tests.paged_ref import Pool

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


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(ham, s):
    return torch.full((ham.ham_op_paged_workspace_bytes(s),), 0x5A, dtype=torch.uint8, device=DEV)


def rows_of_pages(ham, dtype, H, Hk, hd, P, lens, spare=3, seed=11, n_pages=None):
    """A pool whose rows hold `lens` slots of N(0, 1) in pages of no order, everything else bytes 0xFF (NaN)."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // P) for n in lens]
    s = ham.paged_shape(dtype, len(lens), H, Hk, hd, P, n_pages or sum(need) + spare, max(need) + 1)
    pool = Pool(s, fill=0xFF)
    ids = torch.randperm(s.n_pages, generator=g).tolist()
    for r, n in enumerate(lens):
        pool.len[r] = n
        pool.table[r][:need[r]] = [ids.pop() for _ in range(need[r])]
        for p in pool.table[r][:need[r]]:
            pool.refs[p] += 1
        if n:
            pool.append(r, 0, *(stored(torch.randn(n, Hk, hd, generator=g).double(), dtype) for _ in range(2)))
    return s, pool, g


def queries(g, n, H, hd, dtype, sigma=1.0):
    """Act rows on the CPU and what they stand for, float64 [n][H][hd]."""
    q = act_rows(torch, sigma * torch.randn(n, H * hd, generator=g), dtype)
    return q, from_act(torch, q, H * hd, dtype).double().view(n, H, hd)


def values(out, H, hd, dtype):
    return from_act(torch, out, H * hd, dtype).double().cpu().view(-1, H, hd)


def attend(ham, s, pool, q, lens, kv_max=None, enable=None, table=None):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    err = i32([0] * s.rows)
    ham.ham_op_paged_attention(s, q.to(DEV), pool.data.to(DEV), i32(table or pool.table), i32(lens), i32(enable or [1] * s.rows),
                               max(lens) if kv_max is None else kv_max, out, err, workspace(ham, s), stream())
    return values(out, s.n_heads, s.head_dim, s.dtype), err.tolist()


def prompt(ham, s, pool, q, offsets, lens, kv_max=None, table=None):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    err = i32([0] * s.rows)
    ham.ham_op_paged_prompt(s, q.to(DEV), i32(offsets), pool.data.to(DEV), i32(table or pool.table), i32(lens),
                            max(lens) if kv_max is None else kv_max, out, err, workspace(ham, s), stream())
    return out.cpu(), err.tolist()


def near(got, want, dtype):
    """Largest difference of a (row, q-head) over the root mean square of its output."""
    rms = want.square().mean(-1).sqrt()
    worst = ((got - want).abs().amax(-1) / rms.clamp(min=1e-30))[rms > 0]
    assert worst.numel() == 0 or worst.max() < FILLED_TOL[dtype], worst.max()
    assert torch.all(got[rms == 0] == 0)


# ---------------------------------------------------------------- append
# dtype, q-heads, kv heads, head dim, page, slots held, new tokens
APPENDS = [
    (BF16, 32, 8, 64, 32, [700], [1]), (BF16, 32, 8, 128, 16, [0, 31, 32, 63, 5], [1, 1, 1, 1, 0]), (F32, 4, 2, 64, 16, [0], [64]),
    (BF16, 9, 3, 64, 32, [30, 0, 33, 64], [37, 70, 31, 0]), (F32, 8, 8, 128, 64, [17], [100]), (BF16, 16, 1, 128, 256, [40, 1], [33, 300]),
    (BF16, 4, 4, 64, 128, [95, 96, 97], [2, 33, 128]), (F32, 5, 5, 64, 32, [31, 3], [33, 2]), (BF16, 2, 1, 64, 16, [13], [22]),
    (BF16, 8, 2, 128, 16, list(range(40)), [1] * 40), (F32, 3, 1, 128, 16, list(range(70)), [i % 4 for i in range(70)]),
    (BF16, 4, 2, 64, 64, [7] * 130, [i % 3 for i in range(130)])]


@pytest.mark.parametrize("dtype,H,Hk,hd,P,start,count", APPENDS)
def test_append_writes_what_it_says_and_nothing_else(ham, dtype, H, Hk, hd, P, start, count):
    R = len(start)
    s, pool, g = rows_of_pages(ham, dtype, H, Hk, hd, P, [a + b for a, b in zip(start, count)])
    before, behind = 2, 3   # packed rows that belong to no sequence
    offsets = [before]
    for c in count:
        offsets.append(offsets[-1] + c)
    N = offsets[-1] + behind
    qkv, a = torch.randn(N, H + 2 * Hk, hd, generator=g), 6.28 * torch.rand(N, hd // 2, generator=g)
    cos, sin = a.cos(), a.sin()
    dev = pool.data.to(DEV)
    q = torch.full((N, H * hd * (2 if dtype == BF16 else 1)), 7.0, dtype=storage(dtype), device=DEV)
    err = i32([0] * R)

    def run(q):
        ham.ham_op_paged_append(s, qkv.view(N, -1).to(DEV), cos.to(DEV), sin.to(DEV), i32(offsets), i32(start), i32(pool.table), dev, q, err,
                                stream())
    run(q)
    rot = rope64(qkv[:, :H + Hk].double(), cos.double()[:, None], sin.double()[:, None])
    k, v = stored(rot[:, H:], dtype), stored(qkv[:, H + Hk:].double(), dtype)
    want_q = torch.full(q.shape, 7.0, dtype=torch.float64)
    for r in range(R):
        i = slice(offsets[r], offsets[r + 1])
        pool.append(r, start[r], k[i], v[i])
        want_q[i] = act64(rot[i, :H].reshape(count[r], H * hd), dtype)
    bits = torch.int16 if dtype == BF16 else torch.int32
    assert torch.equal(dev.cpu().view(bits), pool.data.view(bits))
    assert torch.equal(q.cpu().double(), want_q) and err.tolist() == [0] * R
    dev.copy_(rows_of_pages(ham, dtype, H, Hk, hd, P, [a + b for a, b in zip(start, count)])[1].data)   # without q: the same pool
    run(None)
    assert torch.equal(dev.cpu().view(bits), pool.data.view(bits)) and err.tolist() == [0] * R


def test_append_that_does_not_fit_writes_nothing(ham):
    s, pool, g = rows_of_pages(ham, BF16, 4, 2, 64, 16, [40, 40, 40, 40])
    cap = s.row_pages * 16
    qkv, cs = torch.randn(9, 512, generator=g).to(DEV), torch.ones(9, 32, device=DEV)
    for start, offsets, bad in (([-1, cap, 5, 0], [0, 2, 3, 5, 5], [8, 8, 0, 0]), ([0] * 4, [0, 3, 1, 2, 9], [0, 8, 0, 0]),
                                ([0] * 4, [-2, 1, 1, 1, 10], [8, 0, 0, 8]), ([2147483647] * 4, [0, 1, 2, 3, 4], [8] * 4)):
        dev, err = pool.data.to(DEV), i32([0] * 4)
        q = torch.full((9, 512), 7.0, dtype=torch.bfloat16, device=DEV)
        ham.ham_op_paged_append(s, qkv, cs, cs, i32(offsets), i32(start), i32(pool.table), dev, q, err, stream())
        assert err.tolist() == bad
        for r in range(4):
            pages = pool.table[r][:3]
            if bad[r]:
                assert torch.equal(dev[:, pages].cpu().view(torch.int16), pool.data[:, pages].view(torch.int16)), r


@pytest.mark.parametrize("dtype,count", [(BF16, [i % 3 for i in range(1300)]), (F32, [0] * 1100 + [40, 0, 1] * 30), (BF16, [1] * 257),
                                         (BF16, [0] * 4095 + [70])])
def test_append_of_hundreds_of_rows(ham, dtype, count):
    start = [i % 37 for i in range(len(count))]
    test_append_writes_what_it_says_and_nothing_else(ham, dtype, 6, 3, 64, 16, start, count)


# ---------------------------------------------------------------- attention of one token
# dtype, q-heads, kv heads, head dim, page, slots of each row
ATTENTION = [
    (BF16, 32, 8, 64, 32, [700]), (BF16, 32, 8, 128, 16, [1, 0, 15, 16, 17, 31, 32, 33]), (BF16, 32, 8, 128, 64, [4097, 1]),
    (F32, 4, 2, 64, 16, [1, 2, 15, 16, 17, 100]), (BF16, 16, 1, 128, 256, [3000, 257, 255]), (BF16, 9, 3, 64, 32, [2000, 40, 1999, 65]),
    (F32, 32, 8, 128, 32, [511, 513, 700]), (F32, 16, 1, 64, 128, [9000, 5]), (BF16, 8, 8, 128, 16, [700] * 40), (BF16, 5, 1, 64, 16, [33000]),
    (BF16, 7, 7, 128, 32, [300, 20000]), (BF16, 8, 2, 64, 32, [9000] + [3, 0, 500] * 30), (F32, 2, 2, 64, 16, [4000, 33] * 40), (BF16, 32, 8, 128, 32, [4096] + [70] * 70), (F32, 3, 3, 128, 16, [2500, 0, 16])]


@pytest.mark.parametrize("dtype,H,Hk,hd,P,lens", ATTENTION)
def test_attention_of_one_token(ham, dtype, H, Hk, hd, P, lens):
    s, pool, g = rows_of_pages(ham, dtype, H, Hk, hd, P, lens)
    q, qd = queries(g, len(lens), H, hd, dtype)
    got, err = attend(ham, s, pool, q, lens)
    near(got, pool.attention(qd, lens)[0], dtype)
    assert err == [0] * len(lens)


def test_a_long_row_among_hundreds(ham):
    lens = [i % 50 for i in range(330)]
    lens[200] = 17000
    test_attention_of_one_token(ham, BF16, 4, 2, 128, 32, lens)


@pytest.mark.parametrize("dtype,H,Hk,hd,P,lens", [(BF16, 32, 8, 128, 32, [33, 700, 5000]), (BF16, 16, 1, 64, 16, [200, 3000]),
                                                  (F32, 8, 2, 128, 64, [40, 1500]), (F32, 4, 4, 64, 16, [300])])
def test_no_bf16_plane_of_one_token_is_lost(ham, dtype, H, Hk, hd, P, lens):
    s, pool, g = rows_of_pages(ham, dtype, H, Hk, hd, P, lens)
    q, qd = queries(g, len(lens), H, hd, dtype, kv8_planes.SIGMA_Q)
    got, _ = attend(ham, s, pool, q, lens)
    assert kv8_planes.errors(got, *pool.attention(qd, lens), dtype).max() < 1.0


def test_rows_switched_off_or_out_of_range_are_zero(ham):
    lens = [100, 200, 300, 64, 50]
    s, pool, g = rows_of_pages(ham, BF16, 8, 2, 64, 32, lens)
    q, qd = queries(g, 5, 8, 64, BF16)
    got, err = attend(ham, s, pool, q, [100, 200, -3, 64, 301], kv_max=300, enable=[1, 0, 1, 5, 1])
    want = pool.attention(qd, [100, 0, 0, 64, 0])[0]
    near(got, want, BF16)
    assert err == [0, 0, 8, 0, 8] and torch.all(got[[1, 2, 4]] == 0)
    assert torch.all(attend(ham, s, pool, q, [0] * 5, kv_max=0)[0] == 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_minus_infinity_and_large_ones(ham, dtype):
    lens = [70, 70, 70]
    s, pool, g = rows_of_pages(ham, dtype, 2, 1, 64, 16, lens)
    q = torch.full((3, 128), 2.0 ** 70)       # products and sums overflow
    q[2] = 1e4
    q = act_rows(torch, q, dtype)
    k, v = pool.keys_values(0, 70)
    pool.append(0, 0, torch.full((70, 1, 64), -2.0 ** 70, dtype=torch.float64), v.transpose(0, 1))
    k.zero_()
    k[:, 33:] = -2.0 ** 70
    pool.append(1, 0, k.transpose(0, 1), v.transpose(0, 1))
    qd = from_act(torch, q, 128, dtype).double().view(3, 2, 64)
    got, err = attend(ham, s, pool, q, lens)
    assert torch.all(got[0] == 0) and err == [0, 0, 0]
    want = pool.attention(qd, [0, 70, 70])[0]
    near(got[1:], want[1:], dtype)
    got, _ = prompt(ham, s, pool, q, [0, 1, 2, 3], lens)
    got = values(got, 2, 64, dtype)
    assert torch.all(got[0] == 0)
    near(got[1:], want[1:], dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_an_infinite_key_reaches_the_rows_that_see_it_and_no_other(ham, dtype):
    lens = [70, 70, 70]
    s, pool, g = rows_of_pages(ham, dtype, 2, 1, 64, 16, lens)
    q, qd = queries(g, 3, 2, 64, dtype)
    want = pool.attention(qd, lens)[0]
    k, v = pool.keys_values(1, 70)
    k[:, 33:] = -INF
    pool.append(1, 0, k.transpose(0, 1), v.transpose(0, 1))
    for got, err in (attend(ham, s, pool, q, lens), prompt(ham, s, pool, q, [0, 1, 2, 3], lens)):
        got = got if got.dim() == 3 else values(got, 2, 64, dtype)
        near(got[[0, 2]], want[[0, 2]], dtype)
        assert torch.isnan(got[1]).all() and err == [0, 0, 0]


def test_a_bad_page_is_reported_and_read_nowhere_else(ham):
    lens = [100, 100, 100]
    for dtype in (BF16, F32):
        s, pool, g = rows_of_pages(ham, dtype, 4, 2, 64, 16, lens)
        pool.data.nan_to_num_()
        q, qd = queries(g, 3, 4, 64, dtype)
        table = [list(t) for t in pool.table]
        table[0][2], table[2][6] = s.n_pages, -1
        table[1][7] = 1 << 30          # behind the row's slots: not read
        want = pool.attention(qd, lens)[0]
        for got, err in (attend(ham, s, pool, q, lens, table=table), prompt(ham, s, pool, q, [0, 1, 2, 3], lens, table=table)):
            got = got if got.dim() == 3 else values(got, 4, 64, dtype)
            assert err == [32, 0, 32]
            near(got[1:2], want[1:2], dtype)


# ---------------------------------------------------------------- prompts
# dtype, q-heads, kv heads, head dim, page, (slots held before, tokens) of each row
PROMPTS = [
    (BF16, 32, 8, 64, 32, [(0, 512)]), (BF16, 32, 8, 128, 16, [(0, 1), (5, 1), (16, 3), (0, 0), (100, 65), (0, 64)]),
    (BF16, 8, 8, 128, 64, [(0, 257), (300, 31)]), (BF16, 9, 3, 64, 32, [(40, 70), (0, 333), (1, 1)]), (BF16, 16, 1, 128, 256, [(1000, 40)]),
    (BF16, 5, 1, 64, 16, [(0, 100), (33, 13)]), (BF16, 7, 7, 64, 128, [(200, 300), (0, 129)]), (BF16, 4, 2, 128, 32, [(6000, 3)]),
    (BF16, 32, 8, 128, 32, [(10, 1)] * 70 + [(0, 40)]), (BF16, 6, 1, 128, 16, [(0, 700)]), (BF16, 1, 1, 64, 16, [(0, 1)]),
    (BF16, 16, 1, 64, 64, [(31, 33), (20000, 2)]), (BF16, 32, 8, 64, 32, [(0, 1100), (50, 900), (0, 77)]),
    # enough tokens for the kernel of long prompts: every group size, page size and form of it, splits, rows past the 64th
    (BF16, 16, 1, 128, 256, [(1000, 2100)]), (BF16, 9, 3, 64, 32, [(40, 1900), (0, 1800), (1, 1)]), (BF16, 5, 1, 64, 16, [(0, 3300), (33, 3300)]),
    (BF16, 7, 7, 64, 128, [(200, 2500), (0, 2300)]), (BF16, 8, 8, 128, 64, [(0, 4200)]), (BF16, 32, 8, 128, 32, [(10, 9)] * 70 + [(0, 500)]),
    (BF16, 32, 8, 128, 16, [(0, 1), (5, 1), (16, 3), (0, 0), (100, 65), (0, 64), (0, 1000)]), (BF16, 32, 8, 128, 64, [(33000, 64)]),
    (BF16, 16, 1, 64, 16, [(20000, 40), (17000, 130)]), (BF16, 32, 8, 128, 32, [(5000, 1), (0, 1200), (33, 8), (700, 9), (0, 0), (31, 2)]), (BF16, 12, 1, 128, 32, [(0, 2800)]), (BF16, 32, 8, 128, 32, [(0, 300)] * 20),
    (F32, 4, 2, 64, 16, [(0, 64)]), (F32, 8, 8, 128, 32, [(3, 40), (0, 0), (0, 17), (90, 1)]), (F32, 9, 3, 128, 64, [(0, 130), (500, 20)]),
    (F32, 16, 1, 64, 256, [(700, 9)]), (F32, 5, 1, 128, 16, [(0, 33), (4000, 2)]), (F32, 32, 8, 64, 16, [(2, 3)] * 66)]


def packed(rows, gap=2):
    offsets = [gap]
    for _, c in rows:
        offsets.append(offsets[-1] + c)
    return offsets, [a + b for a, b in rows], offsets[-1] + gap


@pytest.mark.parametrize("dtype,H,Hk,hd,P,rows", PROMPTS)
def test_prompts(ham, dtype, H, Hk, hd, P, rows):
    offsets, lens, N = packed(rows)
    s, pool, g = rows_of_pages(ham, dtype, H, Hk, hd, P, lens)
    q, qd = queries(g, N, H, hd, dtype)
    out, err = prompt(ham, s, pool, q, offsets, lens)
    want = pool.prompt(qd, offsets, lens)[0]
    i = slice(offsets[0], offsets[-1])
    near(values(out, H, hd, dtype)[i], want[i], dtype)
    assert err == [0] * len(rows)
    assert torch.all(out[:offsets[0]] == 7) and torch.all(out[offsets[-1]:] == 7)   # packed rows of no sequence


# the long prompts' kernel with workgroups of 8 waves: one round of them behind many slots, two rounds; of 4: many, several rows
@pytest.mark.parametrize("H,Hk,hd,P,rows", [
    (16, 8, 64, 64, [(8000, 2100), (0, 900)]), (16, 8, 128, 16, [(8100, 2100), (33, 1)]), (8, 1, 128, 32, [(9000, 4100)]), (16, 8, 128, 256, [(0, 7000)]),
    (9, 3, 128, 16, [(0, 7300)]), (32, 8, 64, 16, [(5, 400), (0, 420), (0, 0), (70, 380), (31, 411)]), (7, 7, 128, 128, [(0, 8200)]),
    (16, 8, 128, 32, [(2100, 3000)])])
def test_prompts_of_either_number_of_waves(ham, H, Hk, hd, P, rows):
    test_prompts(ham, BF16, H, Hk, hd, P, rows)


@pytest.mark.parametrize("dtype,H,Hk,rows", [
    (BF16, 4, 1, [(i % 20, 9 + i % 4) for i in range(2100)]), (BF16, 2, 2, [(0, 0)] * 1030 + [(50, 3), (0, 17)] * 10), (F32, 3, 1, [(7, i % 3) for i in range(1100)]),
    (BF16, 16, 1, [(0, 0)] * 4000 + [(5000, 3), (100, 1)] * 3)])
def test_prompts_of_hundreds_of_rows(ham, dtype, H, Hk, rows):
    test_prompts(ham, dtype, H, Hk, 64, 16, rows)


@pytest.mark.parametrize("dtype,H,Hk,hd,P,rows", [(BF16, 32, 8, 128, 32, [(0, 200), (300, 40)]), (BF16, 8, 2, 64, 16, [(2000, 9)]),
                                                  (BF16, 32, 8, 64, 32, [(0, 1100)]), (F32, 8, 2, 128, 16, [(30, 50)])])
def test_no_bf16_plane_of_a_prompt_is_lost(ham, dtype, H, Hk, hd, P, rows):
    offsets, lens, N = packed(rows, 0)
    s, pool, g = rows_of_pages(ham, dtype, H, Hk, hd, P, lens)
    q, qd = queries(g, N, H, hd, dtype, kv8_planes.SIGMA_Q)
    out, _ = prompt(ham, s, pool, q, offsets, lens)
    assert kv8_planes.errors(values(out, H, hd, dtype), *pool.prompt(qd, offsets, lens), dtype).max() < 1.0


@pytest.mark.parametrize("dtype,H,Hk,hd,rows", [(BF16, 8, 2, 128, [(0, 200), (50, 70)]), (BF16, 4, 4, 64, [(300, 90), (0, 33)]),
                                                (F32, 8, 2, 64, [(0, 70), (20, 33)]), (BF16, 16, 1, 128, [(0, 20), (64, 40)]),
                                                (BF16, 32, 8, 64, [(300, 1100), (0, 33)]), (BF16, 16, 1, 128, [(30, 2150), (0, 20)]),
                                                (BF16, 32, 8, 128, [(0, 300)] * 20)])
@pytest.mark.parametrize("bad", [float("nan"), INF, -INF])
def test_what_is_not_finite_reaches_the_tokens_that_see_it_and_no_other(ham, dtype, H, Hk, hd, rows, bad):
    offsets, lens, N = packed(rows, 0)
    s, pool, g = rows_of_pages(ham, dtype, H, Hk, hd, 32, lens)
    q, _ = queries(g, N, H, hd, dtype)
    clean, _ = prompt(ham, s, pool, q, offsets, lens)
    for kind in (0, 1):
        held, c = rows[0]
        at = held + c // 2 + 3              # a slot in the middle of the first row's tokens
        good = pool.data.clone()
        k, v = (x[:, at].clone() for x in pool.keys_values(0, at + 1))
        (k, v)[kind][0, 5] = bad
        pool.append(0, at, k[None], v[None])
        out, err = prompt(ham, s, pool, q, offsets, lens)
        pool.data.copy_(good)
        assert err == [0] * len(rows)
        a, b = values(out, H, hd, dtype), values(clean, H, hd, dtype)
        group = slice(0, H // Hk)           # the q-heads of kv head 0
        seen = torch.zeros(N, dtype=torch.bool)
        seen[at - held:c] = True
        assert torch.equal(a[~seen], b[~seen]) and torch.equal(a[:, H // Hk:], b[:, H // Hk:])
        if kind == 1:                       # V: its channel alone, and with the sign where it has one
            x = a[seen][:, group, 5]
            assert torch.isnan(x).all() if bad != bad or dtype == BF16 else (x == bad).all()
            assert torch.isfinite(a[seen][:, group, 6]).all()
        elif bad != bad:
            assert torch.isnan(a[seen][:, group]).all()


@pytest.mark.parametrize("bad", [float("nan"), -INF])
def test_what_is_not_finite_in_workgroups_of_eight_waves(ham, bad):
    test_what_is_not_finite_reaches_the_tokens_that_see_it_and_no_other(ham, BF16, 16, 8, 128, [(0, 7000)], bad)


@pytest.mark.parametrize("dtype,H,rows", [(BF16, 4, [(10, 20), (0, 30), (5, 5), (40, 9)]), (F32, 4, [(10, 20), (0, 30), (5, 5), (40, 9)]),
                                          (BF16, 32, [(10, 1000), (0, 30), (5, 5), (1040, 9)])])
def test_prompt_rows_that_do_not_fit_are_left(ham, dtype, H, rows):
    offsets, lens, N = packed(rows, 0)
    s, pool, g = rows_of_pages(ham, dtype, H, 2, 64, 16, lens)
    q, qd = queries(g, N, H, 64, dtype)
    want, n = pool.prompt(qd, offsets, lens)[0], rows[0][1]
    # fewer slots than tokens, none, more than kv_max
    out, err = prompt(ham, s, pool, q, offsets, [lens[0], 29, -1, lens[3] + 1], kv_max=lens[3])
    assert err == [0, 8, 8, 8] and torch.all(out[n:] == 7)
    near(values(out, H, 64, dtype)[:n], want[:n], dtype)
    out, err = prompt(ham, s, pool, q, [0, n, n - 10, n - 5, N + 1], lens)
    assert err == [0, 8, 0, 8]


def test_a_bad_page_of_a_long_prompt_is_reported(ham):
    rows = [(0, 600), (0, 700)]
    offsets, lens, N = packed(rows, 0)
    s, pool, g = rows_of_pages(ham, BF16, 32, 8, 64, 16, lens)
    pool.data.nan_to_num_()
    q, qd = queries(g, N, 32, 64, BF16)
    table = [list(t) for t in pool.table]
    table[0][20], table[1][44] = -5, 1 << 30       # the second lies behind the row's slots
    out, err = prompt(ham, s, pool, q, offsets, lens, table=table)
    assert err == [32, 0]
    near(values(out, 32, 64, BF16)[600:], pool.prompt(qd, offsets, lens)[0][600:], BF16)


def test_long_prompts_of_scores_of_minus_infinity(ham):
    rows = [(0, 1100), (40, 60)]
    offsets, lens, N = packed(rows, 0)
    s, pool, g = rows_of_pages(ham, BF16, 32, 8, 64, 32, lens)
    k, v = pool.keys_values(1, 100)
    k[:] = -2.0 ** 70
    k[:, 70:] = 0
    pool.append(1, 0, k.transpose(0, 1), v.transpose(0, 1))
    x = torch.randn(N, 2048, generator=g)
    x[1100:] = 2.0 ** 70
    q = act_rows(torch, x, BF16)
    qd = from_act(torch, q, 2048, BF16).double().view(N, 32, 64)
    out, err = prompt(ham, s, pool, q, offsets, lens)
    got, want = values(out, 32, 64, BF16), pool.prompt(qd, offsets, lens)[0]
    assert torch.all(got[1100:1130] == 0) and err == [0, 0]   # tokens at slots 40 .. 69 see such scores alone
    near(got[:1100], want[:1100], BF16)
    near(got[1130:], want[1130:], BF16)


def test_a_prompt_is_what_its_tokens_are_one_by_one(ham):
    for dtype in (BF16, F32):
        rows = [(0, 40), (90, 17)]
        offsets, lens, N = packed(rows, 0)
        s, pool, g = rows_of_pages(ham, dtype, 8, 2, 64, 16, lens)
        q, qd = queries(g, N, 8, 64, dtype)
        out = values(prompt(ham, s, pool, q, offsets, lens)[0], 8, 64, dtype)
        for i in (0, 1, 15, 16):
            got, _ = attend(ham, s, pool, q[[offsets[0] + i, offsets[1] + i]], [rows[0][0] + i + 1, rows[1][0] + i + 1])
            near(out[[offsets[0] + i, offsets[1] + i]], got, dtype)


# ---------------------------------------------------------------- pages
class Books:
    """The reference and the same on the GPU, advanced together."""

    def __init__(self, ham, s, layers, pool=None):
        self.ham, self.s, self.layers = ham, s, layers
        self.ref = pool or Pool(s, layers)
        self.pool = self.ref.data.to(DEV)
        self.kv_len, self.table, self.refs = i32(self.ref.len), i32(self.ref.table), i32(self.ref.refs)
        self.start, self.err, self.ws = i32([-9] * s.rows), i32([0] * s.rows), workspace(ham, s)

    def same(self):
        bits = torch.int16 if self.s.dtype == BF16 else torch.int32
        assert self.kv_len.tolist() == self.ref.len and self.refs.tolist() == self.ref.refs
        assert self.table.tolist() == self.ref.table
        assert torch.equal(self.pool.cpu().view(bits), self.ref.data.view(bits))

    def advance(self, parent, count):
        self.err.zero_()
        self.ham.ham_op_paged_advance(self.s, self.layers, None if parent is None else i32(parent), i32(count), self.kv_len, self.start,
                                      self.table, self.refs, self.pool, self.err, self.ws, stream())
        start, err = self.ref.advance(parent, count)
        assert self.start.tolist() == start and self.err.tolist() == err
        self.same()

    def compact(self):
        n, used = i32([-5] * self.s.n_pages), i32([-5])
        self.ham.ham_op_paged_compact(self.s, self.layers, self.kv_len, self.table, self.refs, self.pool, n, used, self.err, self.ws, stream())
        to, u = self.ref.compact()
        assert n.tolist() == to and used.tolist() == [u]
        self.same()


@pytest.mark.parametrize("dtype,rows,Hk,hd,P,n_pages,row_pages,layers", [
    (F32, 5, 1, 64, 16, 24, 8, 1), (BF16, 12, 2, 64, 32, 90, 12, 3), (BF16, 70, 1, 64, 16, 700, 20, 2), (F32, 3, 3, 128, 16, 40, 30, 1),
    (BF16, 1, 8, 128, 64, 7, 6, 2), (BF16, 2, 1, 64, 16, 1, 1, 1), (BF16, 6, 1, 64, 16, 14, 8, 2)])
def test_random_steps_of_a_scheduler(ham, dtype, rows, Hk, hd, P, n_pages, row_pages, layers):
    g = random.Random(rows)
    s = ham.paged_shape(dtype, rows, Hk, Hk, hd, P, n_pages, row_pages)
    b = Books(ham, s, layers, Pool(s, layers, fill=None))
    b.ref.data.copy_(torch.randn(b.ref.data.shape, generator=torch.Generator().manual_seed(1)))
    b.pool.copy_(b.ref.data)
    refused = forked = 0
    for i in range(60):
        parent = [g.choice((r, r, r, g.randrange(rows), -1)) for r in range(rows)] if g.random() < 0.5 else None
        if g.random() < 0.1 and parent:
            parent[g.randrange(rows)] = g.choice((rows, -2, 1 << 30))
        count = [g.choice((0, 1, 1, 1, 5, P, P + 1, 3 * P, -1, -P, -100000, 1 << 30, -(1 << 31))) for _ in range(rows)]
        b.advance(parent, count)
        assert b.ref.sound()
        refused += 64 in [e & 64 for e in b.err.tolist()]
        forked += any(x > 1 for x in b.ref.refs)
        if i % 9 == 8:
            b.compact()
    assert forked or rows < 3
    assert refused or n_pages != 14        # the pool that the rows outgrow


def test_many_rows_and_pages(ham):
    g = random.Random(2)
    R = 4096
    s = ham.paged_shape(F32, R, 1, 1, 64, 16, 9000, 5)
    b = Books(ham, s, 1)
    b.advance(None, [g.choice((0, 1, 16, 17, 40)) for _ in range(R)])
    b.advance([g.choice((r, r, g.randrange(R), -1)) for r in range(R)], [g.choice((0, 1, 20, -3)) for _ in range(R)])
    b.compact()
    b.advance(list(range(R - 1, -1, -1)), [0] * R)
    b.advance(None, [80] * R)              # no pages left
    assert 64 in b.err.tolist()
    b.advance([0] * R, [1] * R)            # all rows share row 0's pages, then write: one keeps the page


def test_pools_of_many_pages(ham):
    g = random.Random(5)
    R = 300
    b = Books(ham, ham.paged_shape(BF16, R, 1, 1, 64, 16, 36000, 130), 1)
    b.advance(None, [g.choice((0, 1700, 2000, 2033)) for _ in range(R)])
    b.advance([g.choice((r, r, r, -1)) for r in range(R)], [g.choice((0, 1, 40, -300)) for _ in range(R)])   # holes all over, filled from the front
    b.compact()
    b.advance(None, [1] * R)
    b.advance([-1] * 290 + list(range(290, R)), [0] * R)   # the pages of a few rows, far behind
    b.compact()


@pytest.mark.parametrize("rows,row_pages,n_pages", [(4, 1000, 5000), (1000, 4, 3500), (1, 4096, 4100), (5, 819, 4000), (5, 820, 4000)])
def test_rows_that_share_pages_of_tables_of_either_size(ham, rows, row_pages, n_pages):
    g = random.Random(rows)
    b = Books(ham, ham.paged_shape(F32, rows, 1, 1, 64, 16, n_pages, row_pages), 1)
    cap = row_pages * 16
    b.advance(None, [g.randrange(cap // 2) for _ in range(rows)])
    for _ in range(4):
        b.advance([g.choice((r, g.randrange(rows), g.randrange(rows), -1)) for r in range(rows)], [g.choice((0, 1, 17, -5, cap // 3)) for _ in range(rows)])


def test_rows_of_impossible_state_are_left(ham):
    s, pool, g = rows_of_pages(ham, BF16, 2, 1, 64, 16, [20, 30, 40, 0])
    b = Books(ham, s, 1, pool)
    kv, table = list(pool.len), [list(t) for t in pool.table]
    b.kv_len.copy_(i32([20, -7, 1 << 28, 0]))
    b.table[0, 1] = s.n_pages + 5
    refs = b.refs.tolist()
    ham.ham_op_paged_advance(s, 1, i32([0, 1, 2, 2]), i32([3, 3, 3, 3]), b.kv_len, b.start, b.table, b.refs, b.pool, b.err, b.ws, stream())
    # row 0: its last page is bad; rows 1, 2: no length; row 3: a parent without a length, so its own, and three slots
    assert b.err.tolist() == [32, 8, 8, 8] and b.kv_len.tolist() == [23, -7, 1 << 28, 3]
    assert b.table[1:3].tolist() == table[1:3] and kv[3] == 0
    free = refs.index(0)
    assert b.table[3, 0].item() == free and b.refs[free].item() == 1
    n, used = i32([0] * s.n_pages), i32([0])
    b.err.zero_()
    ham.ham_op_paged_compact(s, 1, b.kv_len, b.table, b.refs, b.pool, n, used, b.err, b.ws, stream())
    assert b.err.tolist() == [32, 8, 8, 0] and b.table[1:3].tolist() == table[1:3]


def test_a_caller_keeps_pages_of_its_own(ham):
    # a prompt's pages with one reference more stay when its row is freed, and are taken over by copying its table
    s, pool, g = rows_of_pages(ham, BF16, 2, 1, 64, 16, [40, 0], spare=5)
    b = Books(ham, s, 1, pool)
    kept = pool.table[0][:3]
    for p in kept:
        pool.refs[p] += 1
    b.refs.copy_(i32(pool.refs))
    b.advance([-1, -1], [0, 50])
    assert all(pool.refs[p] == 1 for p in kept) and not set(kept) & set(pool.table[1][:4])
    b.compact()


# ---------------------------------------------------------------- together
class Loop:
    """A decode loop on the device: bookkeeping, append, attention of one layer."""

    def __init__(self, ham, s, N):
        self.ham, self.s = ham, s
        W = s.n_heads * s.head_dim * (2 if s.dtype == BF16 else 1)
        z = lambda *d: torch.zeros(*d, dtype=torch.int32, device=DEV)  # noqa: E731
        self.kv_len, self.start, self.table, self.refs, self.err = z(s.rows), z(s.rows), z(s.rows, s.row_pages) - 1, z(s.n_pages), z(s.rows)
        self.pool = torch.zeros(ham.ham_op_paged_pool_bytes(s), dtype=torch.uint8, device=DEV).view(storage(s.dtype))
        self.q, self.out = (torch.zeros(N, W, dtype=storage(s.dtype), device=DEV) for _ in range(2))
        self.ws = workspace(ham, s)

    def step(self, x, offsets, parent, count, on=None):
        h, s, cap = self.ham, self.s, self.s.row_pages * self.s.page_slots
        h.ham_op_paged_advance(s, 1, parent, count, self.kv_len, self.start, self.table, self.refs, self.pool, self.err, self.ws, stream())
        h.ham_op_paged_append(s, *x, offsets, self.start, self.table, self.pool, self.q, self.err, stream())
        if on is None:
            h.ham_op_paged_prompt(s, self.q, offsets, self.pool, self.table, self.kv_len, cap, self.out, self.err, self.ws, stream())
        else:
            h.ham_op_paged_attention(s, self.q, self.pool, self.table, self.kv_len, on, cap, self.out, self.err, self.ws, stream())


def tokens(g, s, N):
    a = 6.28 * torch.rand(N, s.head_dim // 2, generator=g)
    return [t.to(DEV) for t in (torch.randn(N, (s.n_heads + 2 * s.n_kv_heads) * s.head_dim, generator=g), a.cos(), a.sin())]


def kv_of(x, s):
    """Stored K, V of projection rows, float64."""
    H, Hk = s.n_heads, s.n_kv_heads
    qkv, c, sn = (t.cpu().double() for t in x)
    qkv = qkv.view(-1, H + 2 * Hk, s.head_dim)
    return stored(rope64(qkv[:, H:H + Hk], c[:, None], sn[:, None]), s.dtype), stored(qkv[:, H + Hk:], s.dtype)


@pytest.mark.parametrize("dtype,hd,P", [(BF16, 128, 16), (BF16, 64, 64), (F32, 64, 16)])
def test_prompts_beams_and_decode_steps_captured_and_replayed(ham, dtype, hd, P):
    """Prompts of two searches, two beams each; then steps in which beams go on from others, eager and replayed from a graph that
    shares nothing with the eager loop, checked against a history kept on the CPU."""
    R, H, Hk = 4, 8, 2
    s = ham.paged_shape(dtype, R, H, Hk, hd, P, 60, 200 // P + 2)
    g = torch.Generator().manual_seed(4)
    lens, n = [37, 0, 90, 0], 127
    x0 = tokens(g, s, n)
    k0, v0 = kv_of(x0, s)
    off = [0, 37, 37, 127, 127]
    loops = []
    for _ in range(2):
        a = Loop(ham, s, n)
        a.step(x0, i32(off), None, i32(lens))
        loops.append(a)
    history = [(k0[off[r]:off[r + 1]], v0[off[r]:off[r + 1]]) for r in range(R)]
    parent, count, one, on, offsets = i32([0, 0, 2, 2]), i32([1] * R), i32([1] * R), i32([1] * R), i32(list(range(R + 1)))
    # the same buffers for every step of the graph
    for a in loops:
        a.q, a.out = a.q[:R].clone(), a.out[:R].clone()
    live = [t.clone() for t in tokens(g, s, R)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        loops[1].step(live, offsets, parent, count, on)
    pick = random.Random(9)
    for i in range(40):
        x = tokens(g, s, R)
        p = [0, 0, 2, 2] if i == 0 else [pick.choice((0, 1)), pick.choice((0, 1)), pick.choice((2, 3)), pick.choice((2, 3))]
        parent.copy_(i32(p))
        loops[0].step(x, offsets, parent, one, on)
        for a, b in zip(live, x):
            a.copy_(b)
        graph.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
        k, v = kv_of(x, s)
        history = [(torch.cat([history[p[r]][0], k[r:r + 1]]), torch.cat([history[p[r]][1], v[r:r + 1]])) for r in range(R)]
        for name in ("kv_len", "start", "table", "refs", "err", "q", "out"):
            assert torch.equal(getattr(loops[0], name), getattr(loops[1], name)), (i, name)
        if i % 13 == 0 or i == 39:
            end = loops[0].kv_len.tolist()
            assert end == [len(h[0]) for h in history] and loops[0].err.tolist() == [0] * R
            ref = Pool(ham.paged_shape(dtype, R, H, Hk, hd, P, R * s.row_pages, s.row_pages))
            ref.table = [list(range(r * s.row_pages, (r + 1) * s.row_pages)) for r in range(R)]
            for r in range(R):
                ref.append(r, 0, *history[r])
            qd = values(loops[0].q, H, hd, dtype)
            near(values(loops[0].out, H, hd, dtype), ref.attention(qd, end)[0], dtype)


def test_long_prompts_whose_pages_move(ham):
    """Chunks of two long prompts, appended and attended over in turn with other rows forked, freed and the pool compacted between:
    each call sees the tables that the one before has written; replayed from a graph too."""
    s = ham.paged_shape(BF16, 3, 32, 8, 64, 32, 260, 80)
    g = torch.Generator().manual_seed(14)
    a, x = Loop(ham, s, 1100), [tokens(g, s, 1100) for _ in range(2)]
    off = [i32([0, 1000, 1000, 1100]), i32([0, 30, 30, 1100])]
    counts = [[1000, 0, 100], [30, 0, 1070]]
    lens = [0, 0, 0]
    kv = [[], [], []]
    n, used = i32([0] * s.n_pages), i32([0])
    for step in range(2):
        a.step(x[step], off[step], None, i32(counts[step]))
        k, v = kv_of(x[step], s)
        o = off[step].tolist()
        for r in range(3):
            lens[r] += counts[step][r]
            kv[r].append((k[o[r]:o[r + 1]], v[o[r]:o[r + 1]]))
        first = a.out.clone()
        for parent in ([0, 0, 2], [0, -1, 2]):   # row 1 forks row 0, and is freed
            ham.ham_op_paged_advance(s, 1, i32(parent), i32([0, 5 if parent[1] == 0 else 0, 0]), a.kv_len, a.start, a.table, a.refs, a.pool,
                                     a.err, a.ws, stream())
        ham.ham_op_paged_compact(s, 1, a.kv_len, a.table, a.refs, a.pool, n, used, a.err, a.ws, stream())

        def again():
            ham.ham_op_paged_prompt(s, a.q, off[step], a.pool, a.table, a.kv_len, s.row_pages * 32, a.out, a.err, a.ws, stream())
        a.out.zero_()
        again()
        assert torch.equal(a.out, first) and a.err.tolist() == [0, 0, 0] and a.kv_len.tolist() == lens
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            again()
        for _ in range(3):
            a.out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(a.out, first)
    ref = Pool(ham.paged_shape(BF16, 3, 32, 8, 64, 32, 240, 80))
    ref.table = [list(range(80 * r, 80 * r + 80)) for r in range(3)]
    for r in range(3):
        ref.append(r, 0, torch.cat([t[0] for t in kv[r]]), torch.cat([t[1] for t in kv[r]]))
    want = ref.prompt(values(a.q, 32, 64, BF16), off[1].tolist(), lens)[0]
    near(values(a.out, 32, 64, BF16), want, BF16)


def test_two_streams_read_one_pool(ham):
    lens = [5000, 4000]
    s, pool, g = rows_of_pages(ham, BF16, 32, 8, 128, 32, lens)
    dev, table, n, on = pool.data.to(DEV), i32(pool.table), i32(lens), i32([1, 1])
    qs = [queries(g, 2, 32, 128, BF16)[0].to(DEV) for _ in range(2)]

    def run(q, out, err, ws):
        ham.ham_op_paged_attention(s, q, dev, table, n, on, 5000, out, err, ws, stream())
    bufs = [(torch.zeros_like(q), i32([0, 0]), workspace(ham, s)) for q in qs]
    for q, b in zip(qs, bufs):
        run(q, *b)
    torch.cuda.synchronize()
    want = [b[0].clone() for b in bufs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for b in bufs:
        b[0].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for st, q, b in zip(streams, qs, bufs):
            with torch.cuda.stream(st):
                run(q, *b)
    torch.cuda.synchronize()
    assert all(torch.equal(b[0], w) for b, w in zip(bufs, want))


def test_two_graphs_share_a_workspace(ham):
    lens = [5000, 4000]
    s, pool, g = rows_of_pages(ham, BF16, 8, 2, 64, 16, lens)
    dev, table, n, on, ws = pool.data.to(DEV), i32(pool.table), i32(lens), i32([1, 1]), workspace(ham, s)
    q = [queries(g, m, 8, 64, BF16)[0].to(DEV) for m in (2, 6)]
    out, err, off = [torch.zeros_like(x) for x in q], i32([0, 0]), i32([0, 5, 6])

    def run(i):
        if i == 0:
            ham.ham_op_paged_attention(s, q[0], dev, table, n, on, 5000, out[0], err, ws, stream())
        else:
            ham.ham_op_paged_prompt(s, q[1], off, dev, table, n, 5000, out[1], err, ws, stream())
    want = []
    for i in range(2):
        run(i)
        want.append(out[i].clone())
    graphs, side = [torch.cuda.CUDAGraph() for _ in range(2)], torch.cuda.Stream()
    for i in range(2):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graphs[i], stream=side):
            run(i)
    for k in range(4):
        for i in (0, 1) if k % 2 else (1, 0):
            out[i].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and err.tolist() == [0, 0]


def test_offsets_beyond_32_bits(ham):
    # pages of 1 MB at the end of a pool of 5 GB, written, attended over and copied
    s = ham.paged_shape(BF16, 2, 8, 8, 128, 256, 5000, 3)
    assert ham.ham_op_paged_pool_bytes(s) > 1 << 32
    pool = torch.zeros(5000, 8, 2, 256 * 128, dtype=torch.bfloat16, device=DEV)
    small = Pool(ham.paged_shape(BF16, 2, 8, 8, 128, 256, 6, 3))
    small.table = [[0, 1, 2], [3, 4, 5]]
    table = i32([[4999, 4100, 4998], [4500, 2, 4600]])
    g = torch.Generator().manual_seed(8)
    lens, off = [700, 300], [0, 700, 1000]
    x = tokens(g, s, 1000)
    q, err, ws = torch.zeros(1000, 2048, dtype=torch.bfloat16, device=DEV), i32([0, 0]), workspace(ham, s)
    ham.ham_op_paged_append(s, *x, i32(off), i32([0, 0]), table, pool, q, err, stream())
    k, v = kv_of(x, s)
    for r in range(2):
        small.append(r, 0, k[off[r]:off[r + 1]], v[off[r]:off[r + 1]])
    out = torch.zeros_like(q)
    ham.ham_op_paged_prompt(s, q, i32(off), pool, table, i32(lens), 700, out, err, ws, stream())
    qd = values(q, 8, 128, BF16)
    near(values(out, 8, 128, BF16), small.prompt(qd, off, lens)[0], BF16)
    last = q[[699, 999]].contiguous()
    one = torch.zeros_like(last)
    ham.ham_op_paged_attention(s, last, pool, table, i32(lens), i32([1, 1]), 700, one, err, ws, stream())
    near(values(one, 8, 128, BF16), small.attention(qd[[699, 999]], lens)[0], BF16)
    refs = torch.ones(5000, dtype=torch.int32, device=DEV)   # all held but one: the fork's copy goes there
    refs[4700] = 0
    kv, start = i32(lens), i32([0, 0])
    ham.ham_op_paged_advance(s, 1, i32([1, 1]), i32([0, 1]), kv, start, table, refs, pool, err, ws, stream())
    # row 0 gave up its three pages; the lowest free one (4100) holds the copy of the last page of row 1
    assert kv.tolist() == [300, 301] and table.tolist() == [[4500, 2, -1], [4500, 4100, 4600]] and err.tolist() == [0, 0]
    assert torch.equal(pool[4100], pool[2])
