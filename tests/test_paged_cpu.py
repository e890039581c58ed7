"""The operators on a paged KV cache without a GPU: sizes, refusals of every entry point and of the binding, launch rules, and
the reference that the GPU tests hold them to.

Every call here is refused before anything is launched; pointers are numbers that nothing reads.
"""
import ctypes
import os
import random
import subprocess
import tempfile

import pytest
import torch

from paper_2505_20438_amd import ham
from synth.configs import BF16, F32
from tests.paged_ref import Pool, places

GOOD = dict(dtype=BF16, rows=3, n_heads=32, n_kv_heads=8, head_dim=128, page_slots=32, n_pages=400, row_pages=128)
BIG = 1 << 60


def shape(**kw):
    return ham.paged_shape(*dict(GOOD, **kw).values())


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ham.LIB_PATH):
        pytest.skip("libham.so not built")
    return ham.load_library()


CALLS = {   # arguments after the shape, before the stream
    "append": [7, 256, 256, 256, 256, 256, 256, 256, BIG, 256, 256],
    "attention": [256, 256, BIG, 256, 256, 256, 4000, 256, 256, 256, BIG],
    "prompt": [7, 256, 256, 256, BIG, 256, 256, 4000, 256, 256, 256, BIG],
    "advance": [2, 256, 256, 512, 768, 256, 256, 256, BIG, 256, 256, BIG],
    "compact": [2, 256, 256, 256, 256, BIG, 256, 256, 256, 256, BIG]}


def call(lib, name, s, at=None, value=None):
    args = list(CALLS[name])
    if at is not None:
        args[at] = value
    return getattr(lib, "ham_op_paged_" + name)(None if s is None else ctypes.byref(s), *args, None)


BAD_SHAPES = [("dtype", 2), ("dtype", -1), ("rows", 0), ("rows", 4097), ("n_heads", 0), ("n_heads", 30), ("n_heads", 136),
              ("n_heads", 1032), ("n_kv_heads", 0), ("n_kv_heads", 1), ("head_dim", 96), ("head_dim", 32), ("page_slots", 0),
              ("page_slots", 8), ("page_slots", 48), ("page_slots", 512), ("page_slots", -32), ("n_pages", 0), ("n_pages", (1 << 22) + 1),
              ("row_pages", 0), ("row_pages", (1 << 19) + 1), ("row_pages", -1)]


@pytest.mark.parametrize("field,value", BAD_SHAPES)
def test_bad_shapes_have_no_size_and_no_call(lib, field, value):
    s = shape(**{field: value})
    assert ham.ham_op_paged_pool_bytes(s) == 0 and ham.ham_op_paged_workspace_bytes(s) == 0
    for name in CALLS:
        assert call(lib, name, s) == ham.HAM_EINVAL, name


def test_a_null_shape_and_a_table_past_2_28_are_refused(lib):
    assert lib.ham_op_paged_pool_bytes(None) == 0 and lib.ham_op_paged_workspace_bytes(None) == 0
    for name in CALLS:
        assert call(lib, name, None) == ham.HAM_EINVAL
        assert call(lib, name, shape(rows=4096, row_pages=(1 << 16) + 1)) == ham.HAM_EINVAL


@pytest.mark.parametrize("dtype,Hk,hd,P,n", [(BF16, 8, 128, 32, 400), (F32, 2, 64, 16, 1), (BF16, 1, 64, 16, 3), (F32, 3, 128, 256, 77)])
def test_pool_bytes(lib, dtype, Hk, hd, P, n):
    s = shape(dtype=dtype, n_heads=2 * Hk, n_kv_heads=Hk, head_dim=hd, page_slots=P, n_pages=n, row_pages=1)
    assert ham.ham_op_paged_pool_bytes(s) == n * Hk * 2 * P * hd * (2 if dtype == BF16 else 4)
    assert ham.ham_op_paged_workspace_bytes(s) >= 4 * (s.rows * s.row_pages + 3 * n + 4 * s.rows + 2)


def test_places_fill_a_page():
    for P in (16, 32, 256):
        for hd in (64, 128):
            for E in (4, 8):
                for at in places(P, hd, E):
                    assert sorted(at.reshape(-1).tolist()) == list(range(P * hd))


@pytest.mark.parametrize("name,at,value,code", [
    ("append", 0, 0, "EINVAL"), ("append", 0, (1 << 24) + 1, "EINVAL"), ("append", 0, -1, "EINVAL"), ("append", 1, None, "EINVAL"),
    ("append", 1, 260, "EINVAL"), ("append", 2, None, "EINVAL"), ("append", 2, 264, "EINVAL"), ("append", 3, None, "EINVAL"),
    ("append", 4, None, "EINVAL"), ("append", 5, None, "EINVAL"), ("append", 6, None, "EINVAL"), ("append", 7, None, "EINVAL"),
    ("append", 7, 128, "EINVAL"), ("append", 8, 1000, "ENOMEM"), ("append", 9, 8, "EINVAL"), ("append", 10, None, "EINVAL"),
    ("attention", 0, None, "EINVAL"), ("attention", 0, 24, "EINVAL"), ("attention", 1, None, "EINVAL"), ("attention", 1, 16, "EINVAL"),
    ("attention", 2, 9, "ENOMEM"), ("attention", 3, None, "EINVAL"), ("attention", 4, None, "EINVAL"), ("attention", 5, None, "EINVAL"),
    ("attention", 6, -1, "EINVAL"), ("attention", 6, 4097, "EINVAL"), ("attention", 7, None, "EINVAL"), ("attention", 7, 8, "EINVAL"),
    ("attention", 8, None, "EINVAL"), ("attention", 9, None, "EINVAL"), ("attention", 9, 8, "EINVAL"), ("attention", 10, 64, "ENOMEM"),
    ("prompt", 0, 0, "EINVAL"), ("prompt", 0, (1 << 24) + 1, "EINVAL"), ("prompt", 1, None, "EINVAL"), ("prompt", 1, 8, "EINVAL"),
    ("prompt", 2, None, "EINVAL"), ("prompt", 3, None, "EINVAL"), ("prompt", 3, 100, "EINVAL"), ("prompt", 4, 9, "ENOMEM"),
    ("prompt", 5, None, "EINVAL"), ("prompt", 6, None, "EINVAL"), ("prompt", 7, -1, "EINVAL"), ("prompt", 7, 4097, "EINVAL"),
    ("prompt", 8, None, "EINVAL"), ("prompt", 8, 8, "EINVAL"), ("prompt", 9, None, "EINVAL"), ("prompt", 10, None, "EINVAL"),
    ("prompt", 10, 4, "EINVAL"), ("prompt", 11, 64, "ENOMEM"),
    ("advance", 0, 0, "EINVAL"), ("advance", 0, 1025, "EINVAL"), ("advance", 2, None, "EINVAL"), ("advance", 3, None, "EINVAL"),
    ("advance", 4, None, "EINVAL"), ("advance", 4, 512, "EINVAL"), ("advance", 5, None, "EINVAL"), ("advance", 6, None, "EINVAL"),
    ("advance", 7, None, "EINVAL"), ("advance", 7, 8, "EINVAL"), ("advance", 8, 400 * 8 * 2 * 32 * 128 * 2 * 2 - 1, "ENOMEM"),
    ("advance", 9, None, "EINVAL"), ("advance", 10, None, "EINVAL"), ("advance", 11, 64, "ENOMEM"),
    ("compact", 0, 0, "EINVAL"), ("compact", 1, None, "EINVAL"), ("compact", 2, None, "EINVAL"), ("compact", 3, None, "EINVAL"),
    ("compact", 4, None, "EINVAL"), ("compact", 4, 8, "EINVAL"), ("compact", 5, 8, "ENOMEM"), ("compact", 6, None, "EINVAL"),
    ("compact", 7, None, "EINVAL"), ("compact", 8, None, "EINVAL"), ("compact", 9, None, "EINVAL"), ("compact", 10, 64, "ENOMEM")])
def test_refusals(lib, name, at, value, code):
    assert call(lib, name, shape(), at, value) == getattr(ham, "HAM_" + code)
    assert lib.ham_last_error()


def test_calls_past_one_launch_are_refused(lib):
    s = shape(n_heads=1024, n_kv_heads=1024, rows=4096, row_pages=1 << 16, page_slots=16)
    for name in ("append", "prompt"):
        assert call(lib, name, s, 0, 1 << 24) == ham.HAM_EINVAL and b"too large" in lib.ham_last_error()
    s = shape(n_heads=1024, n_kv_heads=1024, n_pages=1 << 22, page_slots=256)
    for name in ("advance", "compact"):
        if name == "advance":
            s = shape(n_heads=1024, n_kv_heads=1024, rows=4096, page_slots=256, row_pages=16)
        args = list(CALLS[name])
        args[0] = 1024
        assert getattr(lib, "ham_op_paged_" + name)(ctypes.byref(s), *[BIG if a == BIG else a for a in args], None) == ham.HAM_EINVAL
        assert b"too large" in lib.ham_last_error()


# ---------------------------------------------------------------- the binding
def tensors():
    s = ham.paged_shape(BF16, 2, 4, 2, 64, 16, 5, 3)
    i32 = lambda *d: torch.zeros(*d, dtype=torch.int32)  # noqa: E731
    pool = torch.zeros(1, 5, 2, 2, 16 * 64, dtype=torch.bfloat16)
    q = torch.zeros(6, 512, dtype=torch.bfloat16)
    ws = torch.zeros(ham.ham_op_paged_workspace_bytes(s), dtype=torch.uint8)
    return s, {
        "append": dict(qkv=torch.zeros(6, 512), cos=torch.zeros(6, 32), sin=torch.zeros(6, 32), offsets=i32(3), start=i32(2), table=i32(2, 3),
                       pool=pool, q=q, err=i32(2), stream=0),
        "attention": dict(q=q[:2], pool=pool, table=i32(2, 3), kv_len=i32(2), enable=i32(2), kv_max=48, out=q[:2], err=i32(2), workspace=ws,
                          stream=0),
        "prompt": dict(q=q, offsets=i32(3), pool=pool, table=i32(2, 3), kv_len=i32(2), kv_max=48, out=q, err=i32(2), workspace=ws, stream=0),
        "advance": dict(n_layers=1, parent=i32(2), count=i32(2), kv_len=i32(2), start=i32(2), table=i32(2, 3), refs=i32(5), pool=pool,
                        err=i32(2), workspace=ws, stream=0),
        "compact": dict(n_layers=1, kv_len=i32(2), table=i32(2, 3), refs=i32(5), pool=pool, map=i32(5), used=i32(1), err=i32(2), workspace=ws,
                        stream=0)}


def test_the_binding_refuses_host_tensors_and_nothing_else_of_good_ones(lib):
    s, calls = tensors()
    for name, kw in calls.items():
        with pytest.raises(ham.HamError, match="on a GPU"):   # host memory never reaches a kernel
            getattr(ham, "ham_op_paged_" + name)(s, **kw)
    for name, key in (("append", "q"), ("advance", "parent")):
        with pytest.raises(ham.HamError, match="on a GPU"):
            getattr(ham, "ham_op_paged_" + name)(s, **dict(calls[name], **{key: None}))


def test_the_binding_refuses_tensors_of_another_size_type_or_stride(lib):
    s, calls = tensors()
    for name, kw in calls.items():
        for key, t in kw.items():
            if not torch.is_tensor(t):
                continue
            bad = [t.double() if key != "workspace" else t[:0][::2]]          # values of another size
            if key != "workspace":
                flat = t.reshape(-1)
                bad += [torch.cat([flat, flat[:1]]), flat[:-1]] + ([torch.stack([t, t], -1)[..., 0]] if t.numel() > 1 else [])
            for x in bad:
                with pytest.raises(ham.HamError) as e:
                    getattr(ham, "ham_op_paged_" + name)(s, **dict(kw, **{key: x}))
                assert e.value.code == ham.HAM_EINVAL and (key == "workspace" or "on a GPU" not in str(e.value)), (name, key)
    for name in ("advance", "compact"):   # a pool of two layers, of which the call names one, and the other way round
        with pytest.raises(ham.HamError, match="pool holds"):
            getattr(ham, "ham_op_paged_" + name)(s, **dict(calls[name], pool=torch.zeros(2, 5, 2, 2, 1024, dtype=torch.bfloat16)))
        with pytest.raises(ham.HamError, match="pool holds"):
            getattr(ham, "ham_op_paged_" + name)(s, **dict(calls[name], n_layers=2))
    for x in (torch.zeros(6, 256, dtype=torch.float32), torch.zeros(6, 512, dtype=torch.float32)):   # rows of the other storage type
        with pytest.raises(ham.HamError):
            ham.ham_op_paged_prompt(s, **dict(calls["prompt"], q=x, out=x))


# ---------------------------------------------------------------- launch rules
@pytest.fixture(scope="module")
def rules():
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_20438_amd", "csrc")
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "r.cpp"), os.path.join(d, "r.so")
        with open(src, "w") as f:
            f.write('#include "launch_rules.h"\nextern "C" {\n'
                    'int split(int R, int H, int Hk, int hd, int kv_max, int block) { return ham::paged_attn_split(R, H, Hk, hd, kv_max, block); }\n'
                    'int shares_of(int R, int Hk) { return ham::paged_attn_shares(R, Hk); }\n'
                    'int tile_splits(long long tiles, int Hk, int kv_max, int block) { return ham::paged_tile_splits(tiles, Hk, kv_max, block); }\n'
                    'int shares(int N, int R, int Hk, int grp, int kv_max) { return ham::paged_prompt_grid(N, R, Hk, grp, kv_max).shares; }\n'
                    'int prompt_splits(int N, int R, int Hk, int grp, int kv_max) { return ham::paged_prompt_grid(N, R, Hk, grp, kv_max).splits; }\n'
                    'int waves(int N, int Hk, int grp, int hd, int kv_max) { return ham::paged_prompt_waves(N, Hk, grp, hd, kv_max); }\n'
                    'int as_tiles(int N, int R, int Hk, int grp, int kv_max) { return ham::paged_prompt_tiles(N, R, Hk, grp, kv_max); }\n'
                    'long long append_steps(long long N, long long R) { return ham::paged_append_steps(N, R); }\n'
                    'int append_groups(int N, int R, int heads) { return ham::paged_append_groups(N, R, heads); }\n'
                    'long long tiles(long long N, long long R, long long grp, long long width) { return ham::paged_tiles(N, R, grp, width); }\n}\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", csrc, src, "-o", out], check=True)
        r = ctypes.CDLL(out)
        r.tiles.argtypes, r.tiles.restype = [ctypes.c_longlong] * 4, ctypes.c_longlong
        r.append_steps.argtypes, r.append_steps.restype = [ctypes.c_longlong] * 2, ctypes.c_longlong
        r.tile_splits.argtypes = [ctypes.c_longlong] + [ctypes.c_int] * 3
        yield r


RECORDS = 1 << 15   # query rows times splits that a workspace has room for


def test_splits_have_work_and_their_records_fit(rules):
    for tiles in (1, 2, 3, 5, 8, 31, 32, 33, 64, 100, 256, 257, 4096):
        for hk, grp in ((1, 1), (1, 16), (2, 2), (3, 3), (8, 4), (8, 16), (32, 1), (64, 16), (1024, 1)):
            for kv in (0, 1, 16, 33, 250, 256, 257, 700, 2560, 33300, 1 << 20, 1 << 24):
                n = rules.tile_splits(tiles, hk, kv, 16)
                assert 1 <= n <= 64
                assert n == 1 or (n - 1) * 8 * 16 < kv              # every split has a block
                assert n == 1 or tiles * hk * n * 16 <= RECORDS
                for hd in (64, 128):
                    if rules.split(tiles, hk * grp, hk, hd, kv, 32):
                        assert kv > 28 * 32 and (tiles + rules.shares_of(tiles, hk)) * hk * grp <= RECORDS


def shares(lens, block, n):
    """The shares of the rows' blocks as the kernel forms them: (row, first block, blocks)."""
    nb = [-(-x // block) for x in lens]
    size = max(-(-sum(nb) // (n - min(len(lens), n // 2))), 8, -(-max(nb) // 64))
    return [(r, i * size, min(size, b - i * size)) for r, b in enumerate(nb) for i in range(max(1, -(-b // size)))], size


def test_shares_of_ragged_rows_fit_the_launch():
    g = random.Random(1)
    for _ in range(5000):
        lens = [g.choice((0, 1, 40, g.randint(0, 3000), g.randint(0, 40000))) for _ in range(g.choice((1, 2, 7, 64, 65, 256)))]
        n = g.choice((1, 4, 32, 85, 256))
        cut, size = shares(lens, 32, n)
        assert len(cut) <= n + len(lens) and max(sum(r == x for r, _, _ in cut) for x in range(len(lens))) <= 64
        for r, x in enumerate(lens):
            assert sum(c for q, _, c in cut if q == r) == -(-x // 32)


def test_prompt_splits_have_work_and_their_records_fit(rules):
    for N in (1, 2, 7, 33, 64, 100, 512, 1000, 2048, 16000):
        for R in (1, 2, 9, 64, 65, 4096):
            for hk, grp in ((1, 1), (1, 16), (2, 2), (3, 3), (8, 4), (8, 16), (32, 1), (1024, 1)):
                for kv in (1, 64, 100, 512, 4000, 33300, 1 << 24):
                    k, n = rules.shares(N, R, hk, grp, kv), rules.prompt_splits(N, R, hk, grp, kv)
                    assert k in (1, 2) and 1 <= n <= 64 and (n == 1 or (n - 1) * 64 < kv)
                    assert n == 1 or rules.tiles(N, R, grp, 256 // k) * hk * n * (256 // k) <= RECORDS


@pytest.mark.parametrize("N,R,Hk,grp,kv,tiles,shares,splits", [
    (64, 1, 8, 4, 64, 1, 2, 1), (512, 1, 8, 4, 512, 1, 2, 2), (1500, 1, 8, 4, 1500, 0, 2, 1), (2048, 1, 8, 4, 32768, 0, 1, 1), (64, 64, 8, 4, 33000, 1, 1, 1),
    (64, 1, 8, 4, 33064, 0, 2, 16), (2100, 1, 1, 16, 3100, 0, 2, 1), (13000, 7, 8, 4, 4900, 0, 1, 1), (4, 1, 8, 4, 8004, 1, 2, 31)])
def test_kernels_of_packed_rows(rules, N, R, Hk, grp, kv, tiles, shares, splits):
    assert rules.as_tiles(N, R, Hk, grp, kv) == tiles
    assert rules.shares(N, R, Hk, grp, kv) == shares and rules.prompt_splits(N, R, Hk, grp, kv) == splits


@pytest.mark.parametrize("N,R,Hk,grp,kv,hd,shares,waves", [
    (2048, 1, 8, 4, 32768, 128, 1, 8), (1500, 1, 8, 4, 17500, 64, 1, 8), (2500, 1, 8, 4, 2500, 128, 1, 4), (4000, 1, 8, 4, 4000, 128, 1, 8),
    (4000, 1, 8, 4, 4000, 64, 1, 4), (1600, 4, 8, 4, 400, 128, 1, 4), (1500, 1, 8, 4, 5500, 128, 1, 4), (1500, 6, 8, 4, 4250, 64, 1, 4), (12452, 7, 8, 4, 4001, 128, 1, 4)])
def test_waves_of_long_prompts(rules, N, R, Hk, grp, kv, hd, shares, waves):
    assert rules.shares(N, R, Hk, grp, kv) == shares and rules.waves(N, Hk, grp, hd, kv) == waves


def test_tiles_do_for_every_cut_of_the_tokens(rules):
    g = random.Random(3)
    for _ in range(20000):
        grp, width = g.randint(1, 16), g.choice((16, 128, 256))
        counts = [g.choice((0, 1, 2, g.randint(0, 200))) for _ in range(g.randint(1, 12))]
        need = sum(-(-c * grp // width) for c in counts)
        assert need <= rules.tiles(max(1, sum(counts)), len(counts), grp, width)


def test_appends_of_many_rows_have_workgroups_for_every_step(rules):
    g = random.Random(4)
    for _ in range(5000):
        rows = [(g.randint(0, 99), g.choice((0, 1, g.randint(0, 200)))) for _ in range(g.randint(1, 200))]
        N = max(1, sum(c for _, c in rows))
        need = sum((s + c - 1) // 32 - s // 32 + 1 for s, c in rows if c)
        assert need <= rules.append_steps(N, len(rows))
    for R in (1, 64, 65, 300, 4096):
        for N in (1, 64, 65, 1000, 5000, 1 << 24):
            for heads in (1, 2, 16, 2048):
                n = rules.append_groups(N, R, heads)
                assert 1 <= n <= heads and (R > 64 or n == heads)


# ---------------------------------------------------------------- the reference
def test_the_reference_keeps_its_books():
    """Random steps of the reference: references match the tables, contents survive, one writer to a page."""
    g = random.Random(5)
    s = ham.paged_shape(F32, 5, 2, 1, 64, 16, 24, 8)
    pool = Pool(s, fill=0)
    want = [[] for _ in range(s.rows)]
    mark = 0.0
    for _ in range(300):
        parent = [g.choice((r, r, r, g.randrange(s.rows), -1)) for r in range(s.rows)] if g.random() < 0.5 else None
        count = [g.choice((0, 1, 1, 5, 17, 40, -1, -7, -20, 500)) for _ in range(s.rows)]
        start, err = pool.advance(parent, count)
        if parent is not None:
            want = [list(want[p]) if p >= 0 else [] for p in parent]
        assert pool.sound() and all(p >= 0 for r in range(s.rows) for p in pool.table[r][:pool.pages(pool.len[r])])
        for r in range(s.rows):
            n = pool.len[r]
            if n < len(want[r]):
                del want[r][n:]
            new = n - len(want[r])
            assert start[r] == len(want[r]) and (new == 0 or not err[r])
            k = torch.zeros(new, 1, 64, dtype=torch.float64)
            for i in range(new):
                mark += 1.0
                k[i] = mark
                want[r].append(mark)
            pool.append(r, start[r], k, -k)
        for r in range(s.rows):
            k, v = pool.keys_values(r, pool.len[r])
            assert k[0, :, 3].tolist() == want[r] and v[0, :, 63].tolist() == [-x for x in want[r]]
        if g.random() < 0.2:
            to, used = pool.compact()
            assert used == sum(x > 0 for x in pool.refs) and all(x > 0 for x in pool.refs[:used]) and pool.sound()
            for r in range(s.rows):
                assert pool.keys_values(r, pool.len[r])[0][0, :, 9].tolist() == want[r]
