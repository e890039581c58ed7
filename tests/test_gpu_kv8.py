"""The operators on a KV cache in 8 bits (``ham_op_kv8_*``) against their definition in float64 (``kv8_ref``; tolerances
there), through the C ABI.

Marked ``gpu``: needs an MI355X and ``libham.so`` built in-tree.
"""
import numpy as np
import pytest
import torch

from synth.configs import BF16, F32
from tests import kv8_planes, kv8_ref
from tests.attention_bounds import FILLED_TOL
from tests.gpu_util import act_rows, from_act, tiled_v
from tests.kv8_ref import B, F8, Cache, act64, rope64, storage, stored

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


def stream():
    return torch.cuda.current_stream().cuda_stream


def new_cache(ham, s, fill=0xAB):
    """A reference cache of bytes 0xAB and the same on the GPU."""
    n = ham.ham_op_kv8_cache_bytes(s)
    ref = Cache(s, ham.ham_op_kv8_info(s), n, torch.full((n,), fill, dtype=torch.uint8))
    return ref, ref.buf.to(DEV)


def tokens(g, s, T):
    """Projection rows and RoPE factors of T tokens per row, on the CPU."""
    H, Hk, hd = s.n_heads, s.n_kv_heads, s.head_dim
    qkv = torch.randn(s.rows, T, H + 2 * Hk, hd, generator=g)
    a = 6.28 * torch.rand(s.rows, T, hd // 2, generator=g)
    return qkv, a.cos(), a.sin()


def append(ham, s, x, start, count, cache, err, q=None):
    ham.ham_op_kv8_append(s, *(t.reshape(s.rows, t.shape[1], -1).contiguous().to(DEV) for t in x), i32(start), i32(count), cache,
                          q, err, stream())


def rotated(x, s):
    """(q, k, v) of tokens as stored or rotated, float64 [rows][T][heads][hd]."""
    qkv, c, sn = (t.double() for t in x)
    rot = rope64(qkv[:, :, :s.n_heads + s.n_kv_heads], c[:, :, None], sn[:, :, None])
    return rot[:, :, :s.n_heads], stored(rot[:, :, s.n_heads:], s.dtype), stored(qkv[:, :, s.n_heads + s.n_kv_heads:], s.dtype)


def valid_equal(a, b, lens):
    """Whether two reference-typed caches hold the same in the slots below each row's length."""
    for r, n in enumerate(lens):
        nb = n // B
        for f in ("codes", "scales", "bounds"):
            assert torch.equal(getattr(a, f)[r, :, :nb], getattr(b, f)[r, :, :nb]), (r, f)
        assert torch.equal(a.open[r, :, :, :n % B], b.open[r, :, :, :n % B]), r


# ---------------------------------------------------------------- writing
# dtype, q-heads, kv heads, head dim, slots held, new slots, tokens of the call
APPENDS = [
    (BF16, 32, 8, 64, [700], [1], 1), (BF16, 32, 8, 128, [0, 31, 32, 63, 5], [1, 1, 1, 1, 0], 1), (BF16, 4, 2, 128, [31], [1], 1),
    (F32, 4, 2, 64, [0], [64], 64), (BF16, 9, 3, 64, [30, 0, 33, 64], [37, 70, 31, 0], 70), (F32, 8, 8, 128, [17], [100], 101),
    (BF16, 16, 1, 128, [40, 1], [33, 300], 300), (BF16, 4, 4, 64, [95, 96, 97], [2, 33, 128], 128), (F32, 5, 5, 64, [31], [33], 65),
    (BF16, 2, 1, 64, [0], [32], 32), (BF16, 2, 1, 64, [10], [22], 22), (BF16, 32, 2, 64, [10, 0], [21, 31], 33)]


@pytest.mark.parametrize("dtype,H,Hk,hd,start,count,T", APPENDS)
def test_append_writes_what_it_says_and_nothing_else(ham, dtype, H, Hk, hd, start, count, T):
    R = len(start)
    s = ham.kv8_shape(dtype, R, H, Hk, hd, (max(a + b for a, b in zip(start, count)) + 31) // 32 * 32)
    ref, cache = new_cache(ham, s)
    g = torch.Generator().manual_seed(5)
    for r in range(R):   # the open block holds what the row has past its last full block
        ref.open[r, :, :, :start[r] % B] = torch.randn(Hk, 2, start[r] % B, hd, generator=g).to(storage(dtype))
    cache.copy_(ref.buf)
    x = tokens(g, s, T)
    q = torch.full((R, T, H * hd * (2 if dtype == BF16 else 1)), 7.0, dtype=storage(dtype), device=DEV)
    err = i32([0] * R)
    append(ham, s, x, start, count, cache, err, q)
    qd, k, v = rotated(x, s)
    want_q = torch.full(q.shape, 7.0, dtype=torch.float64)
    for r in range(R):
        ref.append(r, start[r], k[r, :count[r]], v[r, :count[r]])
        want_q[r, :count[r]] = act64(qd[r, :count[r]].reshape(count[r], H * hd), dtype)
    assert torch.equal(cache.cpu(), ref.buf)
    assert torch.equal(q.cpu().double(), want_q)
    assert err.tolist() == [0] * R
    again = ref.buf.clone()   # without q: the same cache
    append(ham, s, x, start, [0] * R, cache, err, None)
    assert torch.equal(cache.cpu(), again)


@pytest.mark.parametrize("dtype,H,Hk,hd,start,count,T", APPENDS)
def test_append_without_q_writes_the_same_cache(ham, dtype, H, Hk, hd, start, count, T):
    R = len(start)
    s = ham.kv8_shape(dtype, R, H, Hk, hd, (max(a + b for a, b in zip(start, count)) + 31) // 32 * 32)
    ref, cache = new_cache(ham, s)
    g = torch.Generator().manual_seed(15)
    ref.open.copy_(torch.randn(ref.open.shape, generator=g).to(storage(dtype)))
    cache.copy_(ref.buf)
    x, err = tokens(g, s, T), i32([0] * R)
    append(ham, s, x, start, count, cache, err, None)
    _, k, v = rotated(x, s)
    for r in range(R):
        ref.append(r, start[r], k[r, :count[r]], v[r, :count[r]])
    assert torch.equal(cache.cpu(), ref.buf) and err.tolist() == [0] * R


def same(a, b):
    """Equal values (not bits: a zero's sign, a NaN's payload)."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("dtype,hd", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
def test_append_of_extreme_values(ham, dtype, hd):
    # as test_blocks_of_extreme_values; K and V of one head each, in old slots of the open block and in new tokens
    s = ham.kv8_shape(dtype, 1, 4, 2, hd, 32 * 9)
    ref, cache = new_cache(ham, s)
    g = torch.Generator().manual_seed(16)
    ref.open[0, :, :, :20] = torch.randn(2, 2, 20, hd, generator=g).to(storage(dtype))
    ref.open[0, 0, 0, 3, 5] = float("inf")
    ref.open[0, 1, 1, 19, hd - 1] = float("nan")
    cache.copy_(ref.buf)
    qkv, c, sn = tokens(g, s, 250)
    k, v = qkv[0, :, 4:6], qkv[0, :, 6:8]

    def block(b):
        return slice(32 * b - 20, 32 * b + 12)
    k[block(1), 0], v[block(1), 0] = 0, -0.0
    k[block(2)] *= 1e-37
    v[block(2), 1] *= 1e-40
    k[block(3)] *= 5e37
    v[block(3)] *= 1e-30
    k[32 * 4 - 20 + 7, 0, 1] = float("nan")
    v[32 * 4 - 20 + 31, 1, 0] = float("-inf")
    k[32 * 5 - 20, 1, hd // 2] = float("inf")
    v[block(6), 0] = torch.linspace(-1, 1, hd)
    v[32 * 8 - 20 + 2, 0, 9] = float("nan")      # stays in the open block
    k[32 * 8 - 20 + 3, 1, 9] = float("inf")
    x, err = (qkv, c, sn), i32([0])
    append(ham, s, x, [20], [250], cache, err)
    _, k, v = rotated(x, s)
    ref.append(0, 20, k[0], v[0])
    got = Cache(s, ham.ham_op_kv8_info(s), cache.numel(), cache.cpu())
    closed = 270 // B
    scales, want = got.scales[0, :, :closed], ref.scales[0, :, :closed]
    assert same(scales, want)
    assert torch.isnan(want).nonzero().tolist() == [[0, 0, 0], [0, 4, 0], [1, 0, 1], [1, 4, 1], [1, 5, 0]]
    fine = ~torch.isnan(want)
    assert same(got.codes[0, :, :closed][fine].view(F8).float(), ref.codes[0, :, :closed][fine].view(F8).float())
    assert same(got.bounds[0, :, :closed][fine[..., 0]].view(F8).float(), ref.bounds[0, :, :closed][fine[..., 0]].view(F8).float())
    assert same(got.open[0, :, :, :270 % B].float(), ref.open[0, :, :, :270 % B].float()) and err.tolist() == [0]


@pytest.mark.parametrize("dtype,hd,cuts", [(BF16, 128, [1] * 70), (BF16, 64, [31, 1, 2, 36]), (F32, 64, [33, 31, 6]), (BF16, 128, [70])])
def test_the_cache_does_not_depend_on_how_its_slots_arrive(ham, dtype, hd, cuts):
    s = ham.kv8_shape(dtype, 2, 6, 2, hd, 96)
    x = tokens(torch.Generator().manual_seed(6), s, 70)
    one, many = (new_cache(ham, s)[1] for _ in range(2))
    err = i32([0, 0])
    append(ham, s, x, [0, 0], [70, 70], one, err)
    at = 0
    for n in cuts:
        append(ham, s, [t[:, at:at + n] for t in x], [at, at], [n, n], many, err)
        at += n
    info, size = ham.ham_op_kv8_info(s), one.numel()
    valid_equal(Cache(s, info, size, one.cpu()), Cache(s, info, size, many.cpu()), [70, 70])


@pytest.mark.parametrize("start,count", [(-1, 1), (0, -1), (0, 9), (90, 7), (2147483647, 8), (-2147483648, 3)])
def test_append_that_does_not_fit_writes_nothing(ham, start, count):
    s = ham.kv8_shape(BF16, 2, 4, 2, 64, 96)
    ref, cache = new_cache(ham, s)
    x = tokens(torch.Generator().manual_seed(7), s, 8)
    q = torch.full((2, 8, 512), 7.0, dtype=torch.bfloat16, device=DEV)
    err = i32([0, 4])
    append(ham, s, x, [start, 0], [count, 0], cache, err, q)
    assert torch.equal(cache.cpu(), ref.buf) and torch.all(q == 7.0) and err.tolist() == [8, 4]


def test_shortened_rows_go_on(ham):
    # slots of the open block given up, and a row cut to a full block
    s = ham.kv8_shape(BF16, 2, 4, 2, 64, 128)
    g = torch.Generator().manual_seed(8)
    ref, cache = new_cache(ham, s)
    x, y = tokens(g, s, 80), tokens(g, s, 40)
    err = i32([0, 0])
    append(ham, s, x, [0, 0], [80, 80], cache, err)
    append(ham, s, y, [70, 32], [40, 40], cache, err)
    _, k, v = rotated(x, s)
    _, k2, v2 = rotated(y, s)
    for r, n in enumerate((70, 32)):
        ref.append(r, 0, torch.cat([k[r, :n], k2[r]]), torch.cat([v[r, :n], v2[r]]))
    valid_equal(Cache(s, ham.ham_op_kv8_info(s), cache.numel(), cache.cpu()), ref, [110, 72])


@pytest.mark.parametrize("dtype,Hk,hd,lens,S", [(BF16, 8, 128, [100, 0, 32, 31, 65], 128), (F32, 2, 64, [95], 96), (BF16, 3, 64, [64, 1], 160),
                                               (F32, 1, 128, [33, 200], 224)])
def test_pack_writes_what_it_says_and_nothing_else(ham, dtype, Hk, hd, lens, S):
    R = len(lens)
    s = ham.kv8_shape(dtype, R, 2 * Hk, Hk, hd, (max(lens) + 31) // 32 * 32)
    ref, cache = new_cache(ham, s)
    g = torch.Generator().manual_seed(9)
    K, V = (torch.randn(R, Hk, S, hd, generator=g).to(storage(dtype)) for _ in range(2))
    for r in range(R):   # slots past a row's length must not be read
        K[r, :, lens[r]:], V[r, :, lens[r]:] = float("nan"), float("nan")
    err = i32([0] * R)
    ham.ham_op_kv8_pack(s, K.to(DEV), tiled_v(torch, V).to(DEV), i32(lens), max(lens), cache, err, stream())
    for r in range(R):
        ref.append(r, 0, K[r, :, :lens[r]].transpose(0, 1).double(), V[r, :, :lens[r]].transpose(0, 1).double())
    assert torch.equal(cache.cpu(), ref.buf) and err.tolist() == [0] * R


@pytest.mark.parametrize("given", [False, True])
def test_buffers_for_more_rows(ham, given):
    # two of the three rows that every buffer has room for, with the extents taken from the tensors' dimensions or given
    R, H, Hk, hd, S, n = 3, 4, 2, 64, 1024, 5
    s, all_rows = (ham.kv8_shape(BF16, r, H, Hk, hd, S) for r in (2, R))
    g = torch.Generator().manual_seed(14)
    K, V = (torch.randn(R, Hk, S, hd, generator=g).to(torch.bfloat16) for _ in range(2))
    lens = [900, 777]
    ref, cache = new_cache(ham, s)
    vt, err = tiled_v(torch, V).to(DEV), i32([0] * R)
    ham.ham_op_kv8_pack(s, K.to(DEV), vt, i32(lens + [900]), S, cache, err, stream(), S if given else None)
    x = tokens(g, all_rows, 40)
    q = torch.full((R, 40, 2 * H * hd), 7.0, dtype=torch.bfloat16, device=DEV)
    if given:
        ham.ham_op_kv8_append(s, *(t.reshape(R, 40, -1).to(DEV) for t in x), i32(lens + [0]), i32([40, 33, 40]), cache, q, err, stream(), 40)
    else:
        append(ham, s, [t[:2] for t in x], lens, [40, 33], cache, err, q)
    _, k, v = rotated(x, all_rows)
    for r, m in enumerate((40, 33)):
        ref.append(r, 0, K[r, :, :lens[r]].transpose(0, 1).double(), V[r, :, :lens[r]].transpose(0, 1).double())
        ref.append(r, lens[r], k[r, :m], v[r, :m])
    assert torch.equal(cache.cpu(), ref.buf) and torch.all(q[2] == 7.0) and torch.all(q[0] != 7.0) and err.tolist() == [0] * R
    lens = [940, 810]
    qa = act_rows(torch, torch.randn(R, H * hd, generator=g).to(DEV), BF16)
    qd = from_act(torch, qa, H * hd, BF16).double().cpu().view(R, H, hd)[:2]
    blocks, count = (torch.full(d, 77, dtype=torch.int32, device=DEV) for d in ((R, Hk, n), (R, Hk)))
    out, on = torch.full_like(qa, 7.0), i32([1] * R)
    ws = torch.zeros(ham.ham_op_kv8_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    ham.ham_op_kv8_select(s, qa, cache, i32(lens), on, 940, n, 0, 0, blocks, count, err, ws, stream())
    ham.ham_op_kv8_attention(s, qa, cache, i32(lens), on, 940, blocks, count, out, err, ws, stream())
    pairs = [[ref.select(qd, r, h, lens[r], n) for h in range(Hk)] for r in range(2)]
    assert blocks[:2].tolist() == pairs and torch.all(blocks[2] == 77) and torch.all(out[2] == 7.0) and err.tolist() == [0] * R
    near(from_act(torch, out, H * hd, BF16).double().cpu().view(R, H, hd)[:2], ref.attention(qd, lens, pairs), BF16)


def test_pack_of_a_length_out_of_range_writes_nothing(ham):
    s = ham.kv8_shape(BF16, 3, 4, 2, 64, 96)
    ref, cache = new_cache(ham, s)
    K = torch.randn(3, 2, 96, 64, device=DEV).to(torch.bfloat16)
    err = i32([0, 0, 0])
    ham.ham_op_kv8_pack(s, K, tiled_v(torch, K), i32([65, -1, 2147483647]), 64, cache, err, stream())
    assert torch.equal(cache.cpu(), ref.buf) and err.tolist() == [8, 8, 8]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_blocks_of_extreme_values(ham, dtype):
    # zeros, values whose scale is no normal number, the largest and the least ones, an infinity, a NaN: K and V apart
    s = ham.kv8_shape(dtype, 1, 1, 1, 64, 32 * 8)
    ref, cache = new_cache(ham, s)
    g = torch.Generator().manual_seed(10)
    k, v = (torch.randn(256, 1, 64, generator=g) for _ in range(2))
    k[0:32] = 0
    k[32:64] *= 1e-37
    v[32:64] *= 1e-40
    k[64:96] *= 5e37
    v[64:96] *= 1e-30
    k[100, 0, 3] = float("inf")
    v[130, 0, 63] = float("nan")
    k[160:192] = -0.0
    v[192:224, 0] = torch.linspace(-1, 1, 64)
    k, v = k.to(storage(dtype)), v.to(storage(dtype))
    K, V = k.transpose(0, 1)[None].contiguous().to(DEV), tiled_v(torch, v.transpose(0, 1)[None]).to(DEV)
    ham.ham_op_kv8_pack(s, K, V, i32([256]), 256, cache, i32([0]), stream())
    ref.append(0, 0, k.double(), v.double())
    got = Cache(s, ham.ham_op_kv8_info(s), cache.numel(), cache.cpu())
    assert torch.equal(torch.isnan(got.scales), torch.isnan(ref.scales)) and int(torch.isnan(ref.scales).sum()) == 2
    assert torch.equal(torch.nan_to_num(got.scales), torch.nan_to_num(ref.scales))
    fine = ~torch.isnan(ref.scales)
    assert torch.equal(got.codes[fine].view(F8).float(), ref.codes[fine].view(F8).float())
    assert torch.equal(got.bounds[fine[..., 0]].view(F8).float(), ref.bounds[fine[..., 0]].view(F8).float())


# ---------------------------------------------------------------- attention
def filled(ham, dtype, H, Hk, hd, lens, cap=None, seed=11):
    """A cache of random keys and values on CPU and GPU; past each row's length codes, scales and slots are NaN."""
    R = len(lens)
    s = ham.kv8_shape(dtype, R, H, Hk, hd, cap or (max(lens) // 32 + 1) * 32)
    ref, cache = new_cache(ham, s, 0xFF)
    g = torch.Generator().manual_seed(seed)
    for r, n in enumerate(lens):
        nb = n // B
        x = torch.randn(2, Hk, nb, B, hd, generator=g).to(storage(dtype)).double()
        (ck, sk), (cv, sv) = kv8_ref.quantise(x[0]), kv8_ref.quantise(x[1])
        for c, at, j in ((ck, ref.ki, 0), (cv, ref.vi, 1)):
            flat = torch.empty(Hk, nb, B * hd, dtype=torch.uint8)
            flat[..., at.reshape(-1)] = c.view(torch.uint8).reshape(Hk, nb, B * hd)
            ref.codes[r, :, :nb, j] = flat
        ref.scales[r, :, :nb] = torch.stack([sk, sv], -1)
        if nb:
            b = torch.stack([ck.float().amin(2), ck.float().amax(2)], 2).to(F8).view(torch.uint8)
            ref.bounds[r, :, :nb] = b.view(Hk, nb, 2, hd // 8, 8).transpose(2, 3)
        ref.open[r, :, :, :n % B] = torch.randn(Hk, 2, n % B, hd, generator=g).to(storage(dtype))
    cache.copy_(ref.buf)
    q = torch.randn(R, H * hd, generator=g).to(DEV)
    qa = act_rows(torch, q, dtype)
    return s, ref, cache, qa, from_act(torch, qa, H * hd, dtype).double().cpu().view(R, H, hd)


def attend(ham, s, q, cache, lens, kv_max, lists=None, counts=None, enable=None, err=None):
    out = torch.full_like(q, 7.0)
    err = i32([0] * s.rows) if err is None else err
    ws = torch.full((ham.ham_op_kv8_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device=DEV)
    ham.ham_op_kv8_attention(s, q, cache, i32(lens), i32([1] * s.rows if enable is None else enable), kv_max, lists, counts, out, err,
                             ws, stream())
    return from_act(torch, out, s.n_heads * s.head_dim, s.dtype).double().cpu().view(s.rows, s.n_heads, s.head_dim), err.tolist()


def near(got, ref, dtype):
    for r in range(ref.shape[0]):
        for h in range(ref.shape[1]):
            rms = float(ref[r, h].square().mean().sqrt())
            if rms == 0:
                assert torch.all(got[r, h] == 0), (r, h)
            else:
                e = float((got[r, h] - ref[r, h]).abs().max()) / rms
                assert e <= FILLED_TOL[dtype], (r, h, e)


ATTENTIONS = [
    (BF16, 32, 8, 64, [700]), (BF16, 32, 8, 128, [1, 0, 31, 32, 33]), (BF16, 32, 8, 128, [255, 256, 257, 288, 64]),
    (BF16, 4, 4, 64, [1000, 40]), (BF16, 6, 3, 128, [511]), (BF16, 9, 3, 64, [2000, 40, 1999, 65]), (BF16, 10, 2, 64, [333, 2100]),
    (BF16, 32, 4, 128, [1500, 20]), (BF16, 16, 1, 128, [4100, 3]), (BF16, 13, 1, 64, [95]), (F32, 32, 8, 64, [511, 513, 700]),
    (F32, 6, 2, 128, [3001, 0]), (F32, 16, 1, 64, [1, 800]), (F32, 8, 1, 128, [544]), (BF16, 8, 8, 128, [300] * 40),
    (BF16, 32, 8, 128, [4096] + [70] * 16), (BF16, 4, 2, 128, [9000])]


@pytest.mark.parametrize("dtype,H,Hk,hd,lens", ATTENTIONS)
def test_attention_over_every_slot(ham, dtype, H, Hk, hd, lens):
    s, ref, cache, q, qd = filled(ham, dtype, H, Hk, hd, lens)
    want = ref.attention(qd, lens)
    got, err = attend(ham, s, q, cache, lens, max(lens))
    near(got, want, dtype)
    assert err == [0] * len(lens)
    got, err = attend(ham, s, q, cache, lens, s.slots_cap)   # a loose bound: another split
    near(got, want, dtype)


# q-heads to a kv head from 1 to 16: rows of the matrix products that carry the weights' third plane, and none left for it
PLANES = [(BF16, 4, 4, 64), (BF16, 9, 3, 128), (BF16, 8, 2, 128), (BF16, 8, 2, 64), (BF16, 10, 2, 128), (BF16, 16, 2, 64),
          (BF16, 9, 1, 64), (BF16, 13, 1, 128), (BF16, 16, 1, 64), (F32, 4, 4, 64), (F32, 8, 2, 128), (F32, 16, 2, 64), (F32, 16, 1, 128)]


@pytest.mark.parametrize("lens", [[4100, 333], [220, 192]])
@pytest.mark.parametrize("dtype,H,Hk,hd", PLANES)
def test_no_bf16_plane_is_lost(ham, dtype, H, Hk, hd, lens):
    # over every slot, split and not, and over listed blocks
    for pairs in (True, False):
        s, ref, q, qd = kv8_planes.inputs(ham, dtype, H, Hk, hd, lens, pairs)
        q, cache = q.to(DEV), ref.buf.to(DEV)
        some = [[sorted(range(h % 2, n // B, 2)) for h in range(Hk)] for n in lens]
        for lists in (None, some):
            got, err = attend(ham, s, q, cache, lens, max(lens), *((None, None) if lists is None else lists_of(lists, lens[0] // B)))
            part = kv8_planes.errors(got, *kv8_planes.expected(ref, qd, lens, lists), dtype)
            assert float(part.max()) <= 1.0 and err == [0, 0], (pairs, lists is None, part)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_of_1e_30(ham, dtype):
    # weights times V's scale, in three bf16 planes, are normal numbers down to there: errors scale with the values
    lens = [1500, 220]
    s, ref, q, qd = kv8_planes.inputs(ham, dtype, 8, 2, 64, lens, True)
    ref.scales[..., 1] *= 2.0 ** -100
    ref.open[:, :, 1] *= 2.0 ** -100
    got, _ = attend(ham, s, q.to(DEV), ref.buf.to(DEV), lens, 1500)
    part = kv8_planes.errors(got, *kv8_planes.expected(ref, qd, lens), dtype)
    assert float(part.max()) <= 1.0, part


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_minus_infinity(ham, dtype):
    # keys of -infinity in the open block: alone they leave zeros, beside others they count for nothing
    lens = [3, 20, 64 + 5, 31]
    s, ref, cache, q, _ = filled(ham, dtype, 8, 2, 64, lens)
    for r, slots in ((0, 3), (1, 7), (2, 5), (3, 31)):
        ref.open[r, :, 0, :slots] = float("-inf")
    cache.copy_(ref.buf)
    q = act_rows(torch, 0.1 + torch.rand(4, 8 * 64, generator=torch.Generator().manual_seed(17)), dtype).to(DEV)
    qd = from_act(torch, q, 8 * 64, dtype).double().cpu().view(4, 8, 64)
    got, err = attend(ham, s, q, cache, lens, max(lens))
    want = ref.attention(qd, lens)
    assert torch.isnan(want[[0, 3]]).all()   # 0 / 0
    near(got, torch.nan_to_num(want), dtype)
    assert err == [0] * 4


def test_rows_switched_off_or_out_of_range_are_zero(ham):
    lens = [100, 64, 70, 200, 130]
    s, ref, cache, q, qd = filled(ham, BF16, 8, 2, 64, lens)
    got, err = attend(ham, s, q, cache, [100, 64, -1, 1 << 30, 130], 150, enable=[1, 0, 1, 1, 1])
    want = ref.attention(qd, [100, 0, 0, 0, 130])
    near(got, want, BF16)
    assert err == [0, 0, 8, 8, 0]


def lists_of(pairs, n):
    """[row][kv head] lists -> padded device lists and counts."""
    t = torch.full((len(pairs), len(pairs[0]), n), -1, dtype=torch.int32)
    for r, row in enumerate(pairs):
        for h, x in enumerate(row):
            t[r, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
    return t.to(DEV), i32([[len(x) for x in row] for row in pairs])


@pytest.mark.parametrize("dtype,H,Hk,hd,lens,n", [(BF16, 8, 2, 128, [3000, 64, 31, 0, 32], 20), (F32, 4, 2, 64, [1000, 40], 7),
                                                  (BF16, 32, 8, 64, [2100], 65), (BF16, 32, 2, 64, [700, 9000], 100), (BF16, 2, 2, 128, [40000], 1250)])
def test_attention_over_listed_blocks(ham, dtype, H, Hk, hd, lens, n):
    s, ref, cache, q, qd = filled(ham, dtype, H, Hk, hd, lens)
    rng = np.random.default_rng(3)
    pairs = [[sorted(rng.permutation(k // B)[:rng.integers(0, min(n, k // B) + 1)].tolist()) for _ in range(Hk)] for k in lens]
    pairs[0][0] = sorted(rng.permutation(lens[0] // B)[:n].tolist())
    got, err = attend(ham, s, q, cache, lens, max(lens), *lists_of(pairs, n))
    near(got, ref.attention(qd, lens, pairs), dtype)
    assert err == [0] * len(lens)


def test_an_empty_list_leaves_the_open_block_or_nothing(ham):
    lens = [64, 70]
    s, ref, cache, q, qd = filled(ham, BF16, 4, 2, 64, lens)
    pairs = [[[], [1]], [[], []]]
    got, _ = attend(ham, s, q, cache, lens, 70, *lists_of(pairs, 2))
    near(got, ref.attention(qd, lens, pairs), BF16)
    assert torch.all(got[0, :2] == 0) and torch.all(got[1] != 0)


def test_bad_list_entries_are_left_out_and_reported(ham):
    # not ascending, twice the same, negative, at and past the closed blocks; counts out of range
    lens = [1000, 1000, 1000, 1000, 1000, 1000]
    s, ref, cache, q, qd = filled(ham, BF16, 4, 1, 64, lens)
    raw = [[3, 3, 9], [5, 4, 30], [-1, 0, 2], [1, 31, 32], [2, 3, 2147483647], [0, 1, 2]]
    good = [[[3, 9]], [[5, 30]], [[0, 2]], [[1]], [[2, 3]], [[]]]
    blocks, counts = i32(raw).view(6, 1, 3), i32([3, 3, 3, 3, 3, 4]).view(6, 1)
    got, err = attend(ham, s, q, cache, lens, 1000, blocks, counts)
    near(got, ref.attention(qd, lens, good), BF16)
    assert err == [16] * 6
    counts[5] = -1
    got, err = attend(ham, s, q, cache, lens, 1000, blocks, counts)
    near(got, ref.attention(qd, lens, good), BF16)
    assert err == [16] * 6


@pytest.mark.parametrize("kv", [20, 320, 4100])
def test_a_nan_key_or_value_reaches_the_rows_that_read_it_and_no_other(ham, kv):
    lens = [kv] * 4
    s, ref, cache, q, qd = filled(ham, BF16, 8, 2, 64, lens)
    if kv >= B:
        ref.scales[1, 0, kv // B - 1, 0] = float("nan")
        ref.scales[2, 1, 0, 1] = float("nan")
    else:
        ref.open[1, 0, 0, 5, 3] = float("nan")
        ref.open[2, 1, 1, 19, 3] = float("nan")
    cache.copy_(ref.buf)
    got, _ = attend(ham, s, q, cache, lens, kv)
    bad = torch.isnan(got).any(-1)
    assert bad.tolist() == [[False] * 8, [True] * 4 + [False] * 4, [False] * 4 + [True] * 4, [False] * 8]
    for r in (0, 3):
        near(got[r:r + 1], ref.attention(qd, lens)[r:r + 1], BF16)


def test_large_scores(ham):
    # scores of +-1e4: one slot takes everything, no overflow
    s, ref, cache, q, qd = filled(ham, F32, 4, 2, 64, [300, 40])
    q *= 1e3
    got, _ = attend(ham, s, q, cache, [300, 40], 300)
    want = ref.attention(qd * 1e3, [300, 40])
    assert torch.isfinite(got).all()
    # a score of 1e4 has an fp32 error of about 1e4 * 2^-22, and so have the probabilities of slots near the greatest
    assert float((got - want).abs().max()) <= 1e4 * 2.0 ** -22 * 4 * float(want.abs().max())


# ---------------------------------------------------------------- choice of blocks
def choose(ham, s, q, cache, lens, kv_max, n, first=0, last=0, enable=None):
    blocks = torch.full((s.rows, s.n_kv_heads, n), 77, dtype=torch.int32, device=DEV)
    count = torch.full((s.rows, s.n_kv_heads), 77, dtype=torch.int32, device=DEV)
    err = i32([0] * s.rows)
    ws = torch.full((ham.ham_op_kv8_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device=DEV)
    ham.ham_op_kv8_select(s, q, cache, i32(lens), i32([1] * s.rows if enable is None else enable), kv_max, n, first, last, blocks,
                          count, err, ws, stream())
    return blocks, count, err.tolist()


SELECTS = [
    (BF16, 32, 8, 128, [3300, 0, 31, 32, 1000], 16, 0, 0), (BF16, 32, 8, 64, [2560, 2049], 16, 1, 2), (F32, 4, 2, 64, [5000], 7, 3, 4),
    (F32, 16, 1, 128, [700, 40000], 20, 0, 20), (BF16, 9, 3, 64, [1000, 65], 1, 0, 0), (BF16, 5, 1, 128, [1000, 320, 352], 10, 1, 1),
    (BF16, 2, 2, 64, [70000], 1000, 4, 8), (BF16, 5, 1, 64, [300000], 33, 0, 0), (BF16, 4, 1, 64, [4127, 4128, 4160, 4095], 9, 0, 1),
    (BF16, 4, 1, 64, [131071, 131103], 40, 2, 0), (F32, 2, 1, 64, [500000, 4000], 25, 5, 3)]


@pytest.mark.parametrize("dtype,H,Hk,hd,lens,n,first,last", SELECTS)
def test_the_best_blocks_are_chosen(ham, dtype, H, Hk, hd, lens, n, first, last):
    s, ref, cache, q, qd = filled(ham, dtype, H, Hk, hd, lens)
    for kv_max in (max(lens), s.slots_cap):
        blocks, count, err = choose(ham, s, q, cache, lens, kv_max, n, first, last)
        assert err == [0] * len(lens)
        for r, k in enumerate(lens):
            for h in range(Hk):
                want = ref.select(qd, r, h, k, n, first, last)
                assert blocks[r, h].tolist() == want + [-1] * (n - len(want)), (r, h)
                assert int(count[r, h]) == len(want)


def test_equal_scores_take_the_lower_block(ham):
    lens = [B * 2500, B * 50]
    s, ref, cache, q, qd = filled(ham, BF16, 4, 2, 64, lens)
    ref.bounds[:, :, :] = ref.bounds[:, :, :1].clone()     # every block scores alike ...
    ref.scales[:, :, :] = ref.scales[:, :, :1].clone()
    ref.scales[0, :, 7::100] *= 1.0 if float(ref.scores(qd, 0, 0, lens[0])[0]) < 0 else 1.5   # ... or some higher
    ref.bounds[1] = 0                                      # all zero (bounds of +0 and -0 alike)
    ref.bounds[1, :, ::2] = 0x80
    cache.copy_(ref.buf)
    blocks, _, _ = choose(ham, s, q, cache, lens, max(lens), 30, 2, 3)
    for r in range(2):
        for h in range(2):
            assert blocks[r, h].tolist() == ref.select(qd, r, h, lens[r], 30, 2, 3), (r, h)


# lengths around those at which another kernel, more waves or another pass over the keys takes over
EDGES = [([6143, 6144, 4127, 1], 6144, 9, 1, 1), ([6175, 6176, 4128, 5000], 6176, 9, 1, 1), ([65567, 65536, 8223, 8256], 65567, 300, 0, 2),
         ([65568, 65599, 2080, 2111], 65599, 33, 3, 0), ([B * 16384, B * 16387, B * 300], B * 16387, 5, 0, 3),
         ([B * 33000, B * 16390], B * 33000, 260, 2, 1), ([B * 4096, B * 4095], B * 4096, 70, 1, 1),
         ([B * 4097, B * 4096], B * 4097, 70, 1, 1), ([B * 8192, B * 300], B * 8192, 70, 1, 1), ([B * 8193, B * 8192], B * 8193, 70, 1, 1)]


@pytest.mark.parametrize("lens,kv_max,n,first,last", EDGES)
def test_choice_at_the_edges_of_its_rules(ham, lens, kv_max, n, first, last):
    s, ref, cache, q, qd = filled(ham, BF16, 2, 1, 64, lens)
    blocks, count, err = choose(ham, s, q, cache, lens, kv_max, n, first, last)
    assert err == [0] * len(lens)
    for r, k in enumerate(lens):
        want = ref.select(qd, r, 0, k, n, first, last)
        assert blocks[r, 0].tolist() == want + [-1] * (n - len(want)) and int(count[r, 0]) == len(want)


@pytest.mark.parametrize("blocks", [150, 400, 5000, 17000, 40000])
def test_few_distinct_scores(ham, blocks):
    lens = [B * blocks]
    s, ref, cache, q, qd = filled(ham, F32, 1, 1, 64, lens)
    ref.bounds[:, :, :] = ref.bounds[:, :, :1].clone()
    g = torch.Generator().manual_seed(3)
    ref.scales[0, 0, :blocks, 0] = 1.0 + torch.randint(0, 3, (blocks,), generator=g).float()
    cache.copy_(ref.buf)
    for n, first, last in ((1, 0, 0), (blocks // 2, 3, 1), (blocks - 1, 0, 0), (blocks // 3, 0, blocks // 3)):
        got = choose(ham, s, q, cache, lens, lens[0], n, first, last)[0][0, 0].tolist()
        assert got == ref.select(qd, 0, 0, lens[0], n, first, last)


def test_negative_and_nan_scores(ham):
    lens = [B * 1500]
    s, ref, cache, q, qd = filled(ham, F32, 2, 1, 128, lens)
    ref.bounds[:, :, :, :, 1] = ref.bounds[:, :, :, :, 0]      # greatest = least: scores of either sign
    ref.scales[0, 0, [40, 1200], 0] = float("nan")
    cache.copy_(ref.buf)
    got = choose(ham, s, q, cache, lens, lens[0], 900)[0][0, 0].tolist()
    assert got == ref.select(qd, 0, 0, lens[0], 900) and 40 in got and 1200 in got
    assert choose(ham, s, q, cache, lens, lens[0], 2)[0][0, 0].tolist() == [40, 1200]


@pytest.mark.parametrize("dtype,blocks", [(BF16, 20), (BF16, 128), (F32, 192), (BF16, 193), (F32, 1500), (BF16, 5000)])
def test_a_nan_value_is_among_the_chosen_and_seen(ham, dtype, blocks):
    # blocks of which V alone holds a NaN, whose keys score lowest; in one launch (up to 192 blocks) and in two
    lens = [B * blocks + 3, B * blocks]
    s, ref, cache, q, qd = filled(ham, dtype, 4, 2, 64, lens)
    bad = [blocks // 3, blocks - 2]
    ref.scales[0, 1, bad, 1] = float("nan")
    ref.bounds[0, 1, bad] = 0
    ref.bounds[0, 1, bad[0]] = 0x80
    cache.copy_(ref.buf)
    for n in (2, 5):
        chosen, count, err = choose(ham, s, q, cache, lens, max(lens), n)
        for r in range(2):
            for h in range(2):
                assert chosen[r, h].tolist() == ref.select(qd, r, h, lens[r], n), (n, r, h)
        assert set(bad) <= set(chosen[0, 1].tolist()) and err == [0, 0]
        got, _ = attend(ham, s, q, cache, lens, max(lens), chosen, count)
        assert torch.isnan(got).all(-1).tolist() == [[False, False, True, True], [False] * 4]


def test_no_key_of_a_block_left_out_beats_the_least_chosen_score(ham):
    lens = [4000, 1700]
    s, ref, cache, q, qd = filled(ham, BF16, 8, 2, 128, lens)
    blocks, _, _ = choose(ham, s, q, cache, lens, 4000, 12)
    for r, n in enumerate(lens):
        for h in range(2):
            k = ref.keys_values(r, h, n // B * B)[0].view(-1, B, 128)
            best = (k @ qd[r, 4 * h:4 * h + 4].T).amax((1, 2))
            score = ref.scores(qd, r, h, n).double()
            chosen = blocks[r, h].long().cpu()
            left = torch.ones(n // B, dtype=torch.bool)
            left[chosen] = False
            assert torch.all(best[left] <= score[chosen].min() * (1 + 2.0 ** -23)) and torch.all(best <= score + score.abs() * 2.0 ** -23)


@pytest.mark.parametrize("kv_max", [0, 31, 32])
def test_no_closed_block_or_one(ham, kv_max):
    lens = [kv_max, 0]
    s, ref, cache, q, qd = filled(ham, BF16, 8, 2, 64, lens, cap=128)
    blocks, count, err = choose(ham, s, q, cache, lens, kv_max, 3, 1, 1)
    nb = kv_max // B
    assert blocks.tolist() == [[[0] * nb + [-1] * (3 - nb)] * 2, [[-1] * 3] * 2] and count.tolist() == [[nb] * 2, [0] * 2] and err == [0, 0]
    got, err = attend(ham, s, q, cache, lens, kv_max, blocks, count)
    near(got, ref.attention(qd, lens), BF16)
    assert err == [0, 0]


def test_rows_without_a_choice(ham):
    lens = [1000, 1000, 1000]
    s, ref, cache, q, qd = filled(ham, BF16, 4, 2, 64, lens)
    blocks, count, err = choose(ham, s, q, cache, [1000, -5, 1001], 1000, 5, enable=[0, 1, 1])
    assert torch.all(blocks == -1) and torch.all(count == 0) and err == [0, 8, 8]


# ---------------------------------------------------------------- together
def step(ham, s, x, cache, lens, one, on, n, bufs):
    """One decode step: append a token of every row, choose blocks, attend.  Device tensors only."""
    q, blocks, count, out, err, ws = bufs
    ham.ham_op_kv8_append(s, *x, lens, one, cache, q, err, stream())
    lens.add_(one)
    ham.ham_op_kv8_select(s, q, cache, lens, on, s.slots_cap, n, 1, 1, blocks, count, err, ws, stream())
    ham.ham_op_kv8_attention(s, q, cache, lens, on, s.slots_cap, blocks, count, out, err, ws, stream())


@pytest.mark.parametrize("dtype,hd", [(BF16, 128), (F32, 64)])
def test_a_captured_decode_step_replays_as_the_eager_one(ham, dtype, hd):
    R, H, Hk, n = 3, 8, 2, 6
    s = ham.kv8_shape(dtype, R, H, Hk, hd, 640)
    g = torch.Generator().manual_seed(12)
    start = [530, 95, 0]
    x0 = tokens(g, s, 530)
    caches = [new_cache(ham, s)[1] for _ in range(2)]
    for c in caches:
        append(ham, s, x0, [0] * R, start, c, i32([0] * R))
    W = H * hd * (2 if dtype == BF16 else 1)

    def buffers():
        return (torch.zeros(R, W, dtype=storage(dtype), device=DEV), torch.zeros(R, Hk, n, dtype=torch.int32, device=DEV),
                torch.zeros(R, Hk, dtype=torch.int32, device=DEV), torch.zeros(R, W, dtype=storage(dtype), device=DEV), i32([0] * R),
                torch.zeros(ham.ham_op_kv8_workspace_bytes(s), dtype=torch.uint8, device=DEV))
    steps = [[t.reshape(R, 1, -1).to(DEV) for t in tokens(g, s, 1)] for _ in range(40)]
    one, on = i32([1] * R), i32([1] * R)
    lens, bufs = [i32(start) for _ in range(2)], [buffers() for _ in range(2)]
    live = [t.clone() for t in steps[0]]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(ham, s, live, caches[1], lens[1], one, on, n, bufs[1])
    for i, x in enumerate(steps):
        step(ham, s, x, caches[0], lens[0], one, on, n, bufs[0])
        for a, b in zip(live, x):
            a.copy_(b)
        graph.replay()
        if i % 7 == 0:
            torch.cuda.synchronize()
        for a, b in zip(bufs[0][:5], bufs[1][:5]):
            assert torch.equal(a, b), i
    assert lens[0].tolist() == lens[1].tolist() == [k + 40 for k in start] and bufs[0][4].tolist() == [0] * R
    # the last step against the definition, from the tokens
    ref = Cache(s, ham.ham_op_kv8_info(s), caches[0].numel(), torch.zeros(caches[0].numel(), dtype=torch.uint8))
    _, k0, v0 = rotated(x0, s)
    new = [rotated([t.cpu().view(R, 1, *d) for t, d in zip(x, ((H + 2 * Hk, hd), (hd // 2,), (hd // 2,)))], s) for x in steps]
    for r in range(R):
        ref.append(r, 0, torch.cat([k0[r, :start[r]]] + [t[1][r] for t in new]), torch.cat([v0[r, :start[r]]] + [t[2][r] for t in new]))
    qd = from_act(torch, bufs[0][0], H * hd, dtype).double().cpu().view(R, H, hd)
    end = lens[0].tolist()
    pairs = [[ref.select(qd, r, h, end[r], n, 1, 1) for h in range(Hk)] for r in range(R)]
    for r in range(R):
        for h in range(Hk):
            assert bufs[0][1][r, h].tolist() == pairs[r][h] + [-1] * (n - len(pairs[r][h]))
    got = from_act(torch, bufs[0][3], H * hd, dtype).double().cpu().view(R, H, hd)
    near(got, ref.attention(qd, end, pairs), dtype)


def test_two_streams_read_one_cache(ham):
    lens = [5000, 4000]
    s, ref, cache, q, qd = filled(ham, BF16, 32, 8, 128, lens)
    want = attend(ham, s, q, cache, lens, 5000)[0]
    n, on, streams = i32(lens), i32([1, 1]), [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(q) for _ in range(2)]
    spaces = [torch.zeros(ham.ham_op_kv8_workspace_bytes(s), dtype=torch.uint8, device=DEV) for _ in range(2)]
    err = i32([0, 0])
    torch.cuda.synchronize()
    for _ in range(20):
        for st, o, w in zip(streams, outs, spaces):
            ham.ham_op_kv8_attention(s, q, cache, n, on, 5000, None, None, o, err, w, st.cuda_stream)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(from_act(torch, o, 32 * 128, BF16).double().cpu().view(2, 32, 128), want)


def test_a_prefilled_model_state_packs_and_attends(ham):
    # the cache that a prefill leaves in the state buffer, packed; against the attention over the unpacked one
    import synth
    from tests.gpu_util import SMALL16, config_for
    Bt, P, hd, H, Hk = 3, 150, 64, 8, 2
    cfg = config_for(SMALL16, 4, 160, 8)
    rt = ham.HamRuntime(cfg, 21)
    rt.prefill(torch.from_numpy(synth.prompt_ids(22, Bt, P, SMALL16.vocab)).to(DEV), [0] * Bt, i32([1] * Bt))
    info = ham.ham_state_info(cfg, 1)
    S = info["slots"]
    size = 4 * Hk * S * hd * 2
    k, vt = (rt.state[info[o]:info[o] + size].view(torch.bfloat16)[:Bt * Hk * S * hd] for o in ("k_offset", "v_offset"))
    s = ham.kv8_shape(BF16, Bt, H, Hk, hd, S)
    ref, cache = new_cache(ham, s)
    n, err = i32([P, 97, 64]), i32([0] * Bt)
    ham.ham_op_kv8_pack(s, k, vt, n, P, cache, err, stream())
    K, V = (t.double().cpu() for t in rt.kv_cache(1, P))
    lens = n.tolist()
    for r in range(Bt):
        ref.append(r, 0, K[r, :, :lens[r]].transpose(0, 1), V[r, :, :lens[r]].transpose(0, 1))
    assert torch.equal(cache.cpu(), ref.buf)
    q = act_rows(torch, 3.0 * torch.randn(Bt, H * hd, device=DEV), BF16)
    qd = from_act(torch, q, H * hd, BF16).double().cpu().view(Bt, H, hd)
    got, _ = attend(ham, s, q, cache, lens, P)
    near(got, ref.attention(qd, lens), BF16)
    full = torch.zeros_like(q)
    ws = torch.zeros(ham.ham_op_attention_workspace_bytes(Bt, H, Hk, hd), dtype=torch.uint8, device=DEV)
    ham.ham_op_decode_attention(BF16, q, k, vt, n, i32([1] * Bt), P, full, ws, stream(), H, Hk, hd, S)
    full = from_act(torch, full, H * hd, BF16).double().cpu().view(Bt, H, hd)
    for r in range(Bt):
        for h in range(H):
            k8, v8 = ref.keys_values(r, h // 4, lens[r])
            kf, vf = K[r, h // 4, :lens[r]], V[r, h // 4, :lens[r]]
            # |softmax(s + e) - softmax(s)|_1 <= e^(2 max |e|) - 1
            e = float(((k8 - kf) @ qd[r, h]).abs().max()) / hd ** 0.5
            bound = float((v8 - vf).abs().max()) + (np.exp(2 * e) - 1) * float(vf.abs().max())
            assert float((got[r, h] - full[r, h]).abs().max()) <= bound + 1e-3 * float(vf.abs().max()), (r, h)


def test_offsets_beyond_32_bits(ham):
    # codes of 5.4 GB; the last row's last blocks lie beyond 2^32 bytes
    R, H, Hk, hd, cap = 2, 8, 8, 128, (1 << 20) + (1 << 18)
    s = ham.kv8_shape(BF16, R, H, Hk, hd, cap)
    lens = [40, cap - 5]
    cache = torch.empty(ham.ham_op_kv8_cache_bytes(s), dtype=torch.uint8, device=DEV)
    info = ham.ham_op_kv8_info(s)
    g = torch.Generator(device=DEV).manual_seed(13)
    codes = cache[:info["scales"]]
    for i in range(0, codes.numel(), 1 << 28):   # finite codes of both signs, at most 1.875
        part = codes[i:i + (1 << 28)]
        part.copy_(torch.randint(0, 64, part.shape, generator=g, device=DEV, dtype=torch.uint8)
                   + 128 * torch.randint(0, 2, part.shape, generator=g, device=DEV, dtype=torch.uint8))
    nb = cap // B
    scales = cache[info["scales"]:info["scales"] + R * Hk * nb * 8].view(torch.float32).view(R, Hk, nb, 2)
    scales.copy_(0.5 + torch.rand(scales.shape, generator=g, device=DEV))
    bounds = cache[info["bounds"]:info["bounds"] + R * Hk * nb * 2 * hd].view(R, Hk, nb, hd // 8, 2, 8)
    bounds.copy_(torch.randint(0, 64, bounds.shape, generator=g, device=DEV, dtype=torch.uint8))
    bounds[..., 0, :] += 128   # least codes are negative
    opened = cache[info["open"]:info["open"] + R * Hk * 2 * B * hd * 2].view(torch.bfloat16).view(R, Hk, 2, B, hd)
    opened.copy_(torch.randn(opened.shape, generator=g, device=DEV))
    q = act_rows(torch, torch.randn(R, H * hd, generator=g, device=DEV), BF16)
    qd = from_act(torch, q, H * hd, BF16).double().view(R, H, hd)
    # a token into the last row's last block but one slot, at the end of the buffer
    x = [torch.randn(R, 1, (H + 2 * Hk) * hd, generator=g, device=DEV), torch.ones(R, 1, hd // 2, device=DEV), torch.zeros(R, 1, hd // 2, device=DEV)]
    err = i32([0, 0])
    ham.ham_op_kv8_append(s, *x, i32([40, cap - 5]), i32([0, 1]), cache, None, err, stream())
    lens[1] += 1
    assert torch.equal(opened[1, :, 0, 27], x[0][1, 0].view(H + 2 * Hk, hd)[H:H + Hk].to(torch.bfloat16))
    got, e = attend(ham, s, q, cache, lens, cap)
    blocks, count, _ = choose(ham, s, q, cache, lens, cap, 50)
    assert e == [0, 0] and err.tolist() == [0, 0]
    some, _ = attend(ham, s, q, cache, lens, cap, blocks, count)
    ki, vi = (t.to(DEV) for t in kv8_ref.code_index(hd))
    codes = codes.view(R, Hk, nb, 2, B * hd)
    for h in (0, 7):
        n = lens[1] // B
        bd = bounds[1, h, :n].view(F8).double()
        lo, hi = bd[:, :, 0].reshape(-1, hd), bd[:, :, 1].reshape(-1, hd)
        score = (torch.maximum(qd[1, h] * lo, qd[1, h] * hi).sum(-1) * scales[1, h, :n, 0].double()).float()
        want = torch.sort(torch.sort(score, descending=True, stable=True).indices[:50]).values
        assert torch.equal(blocks[1, h].long(), want)
        for at, out in ((torch.arange(n, device=DEV), got), (want, some)):
            c = codes[1, h, at].view(F8)
            k = (c[:, 0].float()[:, ki].double() * scales[1, h, at, 0, None, None].double()).view(-1, hd)
            v = (c[:, 1].float()[:, vi].double() * scales[1, h, at, 1, None, None].double()).view(-1, hd)
            k, v = torch.cat([k, opened[1, h, 0, :lens[1] % B].double()]), torch.cat([v, opened[1, h, 1, :lens[1] % B].double()])
            ref = (torch.softmax(k @ qd[1, h] / hd ** 0.5, 0) @ v).cpu()
            assert float((out[1, h] - ref).abs().max()) <= FILLED_TOL[BF16] * float(ref.square().mean().sqrt()), h


def test_two_graphs_share_a_workspace(ham):
    lens = [20000, 9001]
    s, ref, cache, q, _ = filled(ham, BF16, 16, 2, 64, lens)
    n, on, err = i32(lens), i32([1, 1]), i32([0, 0])
    ws = torch.zeros(ham.ham_op_kv8_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    blocks, count = torch.zeros(2, 2, 30, dtype=torch.int32, device=DEV), torch.zeros(2, 2, dtype=torch.int32, device=DEV)
    out = torch.zeros_like(q)
    calls = [lambda: ham.ham_op_kv8_select(s, q, cache, n, on, 20000, 30, 1, 1, blocks, count, err, ws, stream()),
             lambda: ham.ham_op_kv8_attention(s, q, cache, n, on, 20000, None, None, out, err, ws, stream())]
    graphs, side = [torch.cuda.CUDAGraph() for _ in calls], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for graph, call in zip(graphs, calls):
        with torch.cuda.graph(graph, stream=side):
            call()
    for i in range(6):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
        for call in calls:
            call()
        want = blocks.clone(), count.clone(), out.clone()
        for t in (blocks, count, out):
            t.zero_()
        for graph in (graphs if i % 2 else graphs[::-1]):
            graph.replay()
        for a, b in zip(want, (blocks, count, out)):
            assert torch.equal(a, b), i
    assert err.tolist() == [0, 0]
