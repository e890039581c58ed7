"""The operators on a KV cache in 8 bits without a GPU: sizes, regions, refusals of every entry point, and the launch rule.

Every call here is refused before anything is launched; pointers are numbers that nothing reads.
"""
import ctypes
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2505_20438_amd import ham
from synth.configs import BF16, F32
from tests import kv8_ref

GOOD = dict(dtype=BF16, rows=3, n_heads=32, n_kv_heads=8, head_dim=128, slots_cap=4096)


def shape(**kw):
    s = dict(GOOD, **kw)
    return ham.kv8_shape(*(s[k] for k in ("dtype", "rows", "n_heads", "n_kv_heads", "head_dim", "slots_cap")))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ham.LIB_PATH):
        pytest.skip("libham.so not built")
    return ham.load_library()


BAD_SHAPES = [("dtype", 2), ("dtype", -1), ("rows", 0), ("rows", 4097), ("n_heads", 0), ("n_heads", 30), ("n_heads", 136),
              ("n_kv_heads", 0), ("n_kv_heads", 1), ("head_dim", 96), ("head_dim", 32), ("slots_cap", 0), ("slots_cap", 48),
              ("slots_cap", (1 << 24) + 32), ("slots_cap", -32)]


@pytest.mark.parametrize("field,value", BAD_SHAPES)
def test_bad_shapes_have_no_size_and_no_call(lib, field, value):
    s = shape(**{field: value})
    p = ctypes.byref(s)
    assert ham.ham_op_kv8_cache_bytes(s) == 0 and ham.ham_op_kv8_workspace_bytes(s) == 0
    with pytest.raises(ham.HamError) as e:
        ham.ham_op_kv8_info(s)
    assert e.value.code == ham.HAM_EINVAL
    big = 1 << 60
    assert lib.ham_op_kv8_append(p, 1, 256, 256, 256, 256, 256, 256, big, 256, 256, None) == ham.HAM_EINVAL
    assert lib.ham_op_kv8_pack(p, 256, 256, 4096, 256, 10, 256, big, 256, None) == ham.HAM_EINVAL
    assert lib.ham_op_kv8_select(p, 256, 256, big, 256, 256, 10, 1, 0, 0, 256, 256, 256, 256, big, None) == ham.HAM_EINVAL
    assert lib.ham_op_kv8_attention(p, 256, 256, big, 256, 256, 10, None, None, 0, 256, 256, 256, big, None) == ham.HAM_EINVAL


def test_a_null_shape_is_refused(lib):
    assert lib.ham_op_kv8_cache_bytes(None) == 0 and lib.ham_op_kv8_workspace_bytes(None) == 0
    assert lib.ham_op_kv8_info(None, None, None, None, None) == ham.HAM_EINVAL
    assert lib.ham_op_kv8_info(ctypes.byref(shape()), None, None, None, None) == ham.HAM_EINVAL
    assert lib.ham_op_kv8_append(None, 1, 256, 256, 256, 256, 256, 256, 1 << 60, 256, 256, None) == ham.HAM_EINVAL


@pytest.mark.parametrize("dtype,rows,H,Hk,hd,slots", [(BF16, 3, 32, 8, 128, 4096), (F32, 1, 4, 2, 64, 32), (BF16, 64, 9, 3, 64, 96),
                                                      (BF16, 2, 16, 1, 128, 1 << 24)])
def test_regions_do_not_overlap_and_fit(lib, dtype, rows, H, Hk, hd, slots):
    s = ham.kv8_shape(dtype, rows, H, Hk, hd, slots)
    i, total, blocks = ham.ham_op_kv8_info(s), ham.ham_op_kv8_cache_bytes(s), rows * Hk * slots // 32
    sizes = dict(codes=blocks * 64 * hd, scales=blocks * 8, bounds=blocks * 2 * hd,
                 open=rows * Hk * 64 * hd * (2 if dtype == BF16 else 4))
    spans = sorted((i[k], i[k] + n) for k, n in sizes.items())
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and spans[-1][1] <= total
    assert all(i[k] % 256 == 0 for k in sizes)
    assert ham.ham_op_kv8_workspace_bytes(s) >= blocks * 4


def test_code_positions_fill_a_block():
    for hd in (64, 128):
        for at in kv8_ref.code_index(hd):
            assert sorted(at.reshape(-1).tolist()) == list(range(32 * hd))


# argument positions after the shape; a refused value and the error it gives
@pytest.mark.parametrize("at,value,code", [
    (0, 0, "EINVAL"), (0, (1 << 24) + 1, "EINVAL"), (0, -1, "EINVAL"), (1, None, "EINVAL"), (1, 260, "EINVAL"), (2, None, "EINVAL"), (2, 264, "EINVAL"),
    (3, None, "EINVAL"), (4, None, "EINVAL"), (5, None, "EINVAL"), (6, None, "EINVAL"), (6, 128, "EINVAL"), (7, 1000, "ENOMEM"),
    (8, 8, "EINVAL"), (9, None, "EINVAL")])
def test_append_refusals(lib, at, value, code):
    args = [1, 256, 256, 256, 256, 256, 256, 1 << 60, 256, 256]
    args[at] = value
    assert lib.ham_op_kv8_append(ctypes.byref(shape()), *args, None) == getattr(ham, "HAM_" + code)
    assert lib.ham_last_error()


def test_append_past_one_launch_is_refused(lib):
    s = ham.kv8_shape(BF16, 4096, 32, 8, 128, 1 << 24)
    args = [1 << 20, 256, 256, 256, 256, 256, 256, 1 << 60, 256, 256]
    assert lib.ham_op_kv8_append(ctypes.byref(s), *args, None) == ham.HAM_EINVAL and b"too large" in lib.ham_last_error()


@pytest.mark.parametrize("at,value,code", [
    (0, None, "EINVAL"), (0, 8, "EINVAL"), (1, None, "EINVAL"), (2, 31, "EINVAL"), (2, 0, "EINVAL"), (3, None, "EINVAL"), (4, -1, "EINVAL"),
    (4, 4097, "EINVAL"), (5, None, "EINVAL"), (6, 5, "ENOMEM"), (7, None, "EINVAL")])
def test_pack_refusals(lib, at, value, code):
    args = [256, 256, 8192, 256, 4000, 256, 1 << 60, 256]
    args[at] = value
    assert lib.ham_op_kv8_pack(ctypes.byref(shape()), *args, None) == getattr(ham, "HAM_" + code)


def test_pack_reads_no_slot_that_the_source_lacks(lib):
    assert lib.ham_op_kv8_pack(ctypes.byref(shape()), 256, 256, 64, 256, 65, 256, 1 << 60, 256, None) == ham.HAM_EINVAL


@pytest.mark.parametrize("at,value,code", [
    (0, None, "EINVAL"), (1, None, "EINVAL"), (1, 300, "EINVAL"), (2, 7, "ENOMEM"), (3, None, "EINVAL"), (4, None, "EINVAL"), (5, -1, "EINVAL"),
    (5, 4097, "EINVAL"), (6, 0, "EINVAL"), (6, 129, "EINVAL"), (7, -1, "EINVAL"), (7, 4, "EINVAL"), (8, -1, "EINVAL"), (8, 3, "EINVAL"),
    (8, 2147483647, "EINVAL"), (9, None, "EINVAL"), (10, None, "EINVAL"), (11, None, "EINVAL"), (12, None, "EINVAL"), (13, 64, "ENOMEM")])
def test_select_refusals(lib, at, value, code):
    args = [256, 256, 1 << 60, 256, 256, 4000, 4, 2, 2, 256, 256, 256, 256, 1 << 60]
    args[at] = value
    assert lib.ham_op_kv8_select(ctypes.byref(shape()), *args, None) == getattr(ham, "HAM_" + code)


@pytest.mark.parametrize("at,value,code", [
    (0, None, "EINVAL"), (0, 24, "EINVAL"), (1, None, "EINVAL"), (2, 7, "ENOMEM"), (3, None, "EINVAL"), (4, None, "EINVAL"), (5, -1, "EINVAL"),
    (5, 4097, "EINVAL"), (6, None, "EINVAL"), (7, None, "EINVAL"), (8, 0, "EINVAL"), (8, 129, "EINVAL"), (9, None, "EINVAL"), (9, 8, "EINVAL"),
    (10, None, "EINVAL"), (11, None, "EINVAL"), (12, 64, "ENOMEM")])
def test_attention_refusals(lib, at, value, code):
    args = [256, 256, 1 << 60, 256, 256, 4000, 256, 256, 4, 256, 256, 256, 1 << 60]
    args[at] = value
    assert lib.ham_op_kv8_attention(ctypes.byref(shape()), *args, None) == getattr(ham, "HAM_" + code)


def test_binding_refuses_tensors_that_are_too_small_or_strided(lib):
    s = ham.kv8_shape(BF16, 2, 4, 2, 64, 64)
    i32 = torch.zeros(2, dtype=torch.int32)
    cache = torch.zeros(ham.ham_op_kv8_cache_bytes(s), dtype=torch.uint8)
    ws = torch.zeros(ham.ham_op_kv8_workspace_bytes(s), dtype=torch.uint8)
    q = torch.zeros(2, 512, dtype=torch.bfloat16)
    qkv, cs = torch.zeros(2, 1, 512), torch.zeros(2, 1, 32)

    def attend(**kw):
        a = dict(q=q, cache=cache, kv_len=i32, enable=i32, kv_max=64, blocks=None, count=None, out=q, err=i32, workspace=ws, stream=0)
        ham.ham_op_kv8_attention(s, *dict(a, **kw).values())
    blocks = torch.zeros(2, 2, 1, dtype=torch.int32)
    for bad in (dict(q=q[:, :500]), dict(q=q[:1]), dict(kv_len=i32[:1]), dict(enable=torch.zeros(4, dtype=torch.int32)[::2]),
                dict(out=q[:1]), dict(err=i32[:1]), dict(blocks=blocks, count=blocks[0, :, 0]), dict(blocks=blocks),
                dict(count=blocks), dict(cache=cache[:-256]), dict(workspace=ws[:16])):
        with pytest.raises(ham.HamError):
            attend(**bad)
    with pytest.raises(ham.HamError, match="on a GPU"):   # host memory never reaches a kernel
        attend()
    for bad in (dict(kv_len=i32.long()), dict(enable=i32.long()), dict(err=i32.long()), dict(q=torch.zeros(2, 256)),
                dict(out=torch.zeros(2, 256)), dict(blocks=blocks.long(), count=blocks[:, :, 0].contiguous()),
                dict(blocks=blocks, count=torch.zeros(2, 2, dtype=torch.int64))):
        with pytest.raises(ham.HamError, match="values of"):  # lengths in 64 bits, rows of the other storage type
            attend(**bad)
    for bad in (dict(cos=cs[:1]), dict(sin=cs[:, :, ::2]), dict(start=i32[:1]), dict(q=q[:1]), dict(qkv=qkv[:1])):
        a = dict(qkv=qkv, cos=cs, sin=cs, start=i32, count=i32, cache=cache, q=q, err=i32, stream=0)
        with pytest.raises(ham.HamError):
            ham.ham_op_kv8_append(s, *dict(a, **bad).values())


def host(*dims, dtype=torch.int32):
    return torch.zeros(*dims, dtype=dtype)


def test_binding_refuses_rows_of_another_extent(lib):
    # a call reads row r at r times the extent that its shape gives; where a tensor's rows are longer (a list buffer with room
    # for more blocks, a prompt's q rows), or where its size leaves the extent open (a flat buffer for more rows), it would read
    # other data without an error.  Host tensors: what passes these checks ends with "on a GPU".
    s = ham.kv8_shape(BF16, 2, 4, 2, 64, 64)
    i32, bf = host(2), torch.bfloat16
    cache = host(ham.ham_op_kv8_cache_bytes(s), dtype=torch.uint8)
    ws = host(ham.ham_op_kv8_workspace_bytes(s), dtype=torch.uint8)
    q, W = host(2, 512, dtype=bf), 512

    def attend(**kw):
        a = dict(q=q, cache=cache, kv_len=i32, enable=i32, kv_max=64, blocks=None, count=None, out=q, err=i32, workspace=ws, stream=0)
        ham.ham_op_kv8_attention(s, *dict(a, **kw).values())

    def select(n, **kw):
        a = dict(q=q, cache=cache, kv_len=i32, enable=i32, kv_max=64, n_blocks=n, keep_first=0, keep_last=0, blocks=host(2, 2, n),
                 count=host(2, 2), err=i32, workspace=ws, stream=0)
        ham.ham_op_kv8_select(s, *dict(a, **kw).values())

    def append(n_tokens=None, **kw):
        a = dict(qkv=torch.zeros(2, 3, 512), cos=torch.zeros(2, 3, 32), sin=torch.zeros(2, 3, 32), start=i32, count=i32, cache=cache,
                 q=host(2, 3, 512, dtype=bf), err=i32, stream=0)
        ham.ham_op_kv8_append(s, *dict(a, **kw).values(), n_tokens)

    def pack(src_slots=None, **kw):
        a = dict(k=host(2, 2, 96, 64, dtype=bf), vt=host(2, 2, 3, 64, 32, dtype=bf), kv_len=i32, kv_max=64, cache=cache, err=i32, stream=0)
        ham.ham_op_kv8_pack(s, *dict(a, **kw).values(), src_slots)

    lists, counts = host(2, 2, 2), host(2, 2)
    refused = [
        (attend, dict(q=host(2, 3, W, dtype=bf))), (attend, dict(q=host(2, 2 * W, dtype=bf))), (attend, dict(out=host(3, W + 128, dtype=bf))),
        (attend, dict(blocks=host(3 * 2 * 2), count=counts)), (attend, dict(blocks=host(2, 4), count=counts)),
        (attend, dict(blocks=host(2, 3, 2), count=counts)), (attend, dict(blocks=lists, count=host(2, 3))),
        (select, dict(n=1, blocks=host(2, 2, 2))), (select, dict(n=2, blocks=host(12))), (select, dict(n=1, count=host(2, 3))),
        (append, dict(qkv=torch.zeros(4, 3, 512))), (append, dict(qkv=torch.zeros(6, 512))), (append, dict(qkv=torch.zeros(2, 3, 520))),
        (append, dict(qkv=torch.zeros(2 * 3 * 512))), (append, dict(cos=torch.zeros(2, 4, 32))), (append, dict(sin=torch.zeros(2, 3, 64))),
        (append, dict(q=host(2, 5, 512, dtype=bf))), (append, dict(n_tokens=2)), (append, dict(n_tokens=4)),
        (pack, dict(k=host(4 * 2 * 64 * 64, dtype=bf), vt=host(4 * 2 * 64 * 64, dtype=bf))), (pack, dict(vt=host(2, 2, 4, 64, 32, dtype=bf))),
        (pack, dict(k=host(2, 96, 2, 64, dtype=bf))), (pack, dict(src_slots=64)), (pack, dict(src_slots=192)), (pack, dict(k=host(2, 4, 96, 64, dtype=bf)))]
    for call, kw in refused:
        with pytest.raises(ham.HamError) as e:
            call(**kw)
        assert e.value.code == ham.HAM_EINVAL and "on a GPU" not in str(e.value), (call.__name__, kw.keys(), str(e.value))
    taken = [   # exact sizes whatever the dimensions, and more rows of the same extent
        (attend, {}), (attend, dict(q=host(5, W, dtype=bf), out=host(4, 1, W, dtype=bf), kv_len=host(7), blocks=host(3, 2, 2), count=host(3, 2))),
        (attend, dict(q=host(2 * W, dtype=bf), blocks=lists, count=counts)), (attend, dict(blocks=host(4, 2), count=host(4))),
        (select, dict(n=2)), (select, dict(n=2, blocks=host(5, 2, 2), count=host(5, 2))), (select, dict(n=2, blocks=host(8))),
        (append, {}), (append, dict(qkv=torch.zeros(2, 3, 8, 64), cos=torch.zeros(4, 3, 32), q=None)), (append, dict(q=host(3, 3, 512, dtype=bf))),
        (append, dict(qkv=torch.zeros(6, 512), n_tokens=3)), (append, dict(qkv=torch.zeros(3, 3, 512), n_tokens=3)),
        (append, dict(qkv=torch.zeros(2, 512), cos=torch.zeros(2, 32), sin=torch.zeros(2, 32), q=q)),
        (pack, {}), (pack, dict(k=host(4, 2, 96, 64, dtype=bf), vt=host(4, 2, 3, 64, 32, dtype=bf))), (pack, dict(src_slots=96)),
        (pack, dict(k=host(4, 96, 64, dtype=bf))), (pack, dict(k=host(2, 2, 3, 32, 64, dtype=bf))),
        (pack, dict(k=host(2 * 2 * 64 * 64, dtype=bf), vt=host(2 * 2 * 64 * 64, dtype=bf))),
        (pack, dict(k=host(2 * 2 * 96 * 64, dtype=bf), vt=host(2 * 2 * 96 * 64, dtype=bf), src_slots=96))]
    for call, kw in taken:
        with pytest.raises(ham.HamError, match="on a GPU"):
            call(**kw)


@pytest.fixture(scope="module")
def splits():
    """kv8_attn_splits of csrc/launch_rules.h, compiled on its own."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_20438_amd", "csrc")
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "r.cpp"), os.path.join(d, "r.so")
        with open(src, "w") as f:
            f.write('#include "launch_rules.h"\nextern "C" int splits(int R, int Hk, int hd, int blocks) '
                    '{ return ham::kv8_attn_splits(R, Hk, hd, blocks); }\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", csrc, src, "-o", out], check=True)
        yield ctypes.CDLL(out).splits


def test_split_limits(splits):
    for hd in (64, 128):
        for rows in (1, 2, 3, 7, 16, 33, 64, 500, 4096):
            for hk in (1, 2, 3, 8, 64, 1024):
                for blocks in (0, 1, 7, 8, 16, 17, 33, 64, 80, 100, 512, 1000, 1 << 19):
                    n = splits(rows, hk, hd, blocks)
                    assert 1 <= n <= 64, (rows, hk, blocks)
                    assert n == 1 or n <= 4 or n * 8 < blocks + 8   # a block for every wave
                    assert n >= min(4, blocks // 256)               # a long row among short ones


def test_workspace_holds_the_records_of_every_length(lib, splits):
    for rows, H, hk, hd, slots in ((1, 32, 8, 128, 33344), (4, 32, 8, 128, 33344), (32, 32, 8, 64, 2560), (1, 16, 1, 128, 1 << 20),
                                   (64, 8, 8, 64, 1 << 15), (300, 9, 3, 128, 1 << 16), (4096, 8, 8, 64, 1 << 16)):
        s = ham.kv8_shape(BF16, rows, H, hk, hd, slots)
        for blocks in range(0, slots // 32 + 1, 7):
            n = splits(rows, hk, hd, blocks)
            assert n == 1 or ham.ham_op_kv8_workspace_bytes(s) >= rows * H * n * (hd + 2) * 4


@pytest.mark.parametrize("rows,blocks,n", [(1, 10, 1), (1, 31, 4), (1, 128, 16), (12, 128, 2), (20, 128, 1), (32, 80, 1), (4, 1040, 6), (5, 1040, 5)])
def test_splits_at_eight_heads_of_128(splits, rows, blocks, n):
    assert splits(rows, 8, 128, blocks) == n
