"""The bf16 planes of the weights in the attention over pages: cases on which a lost plane shows, and the kernels' roundings in
float64 with planes to leave out.

The bound is that of kv8_planes.py, KAPPA |S| + OUT |out|, on inputs with pairs: slot 2 i + 1 has the value of slot 2 i with the sign
turned, and nearly its key, so that |out| is a small part of |S| and neither the rounding of the output nor that of long sums hides
the weights'.  (Both slots of a pair enter the same matrix product, so that partial sums stay small too.)  Weights enter in three
planes of the 8 leading bits of what is left, by truncation: 24 bits.  Without the third they lose up to 2^-16 of themselves,
2^-16 / sqrt(12) = 44e-7 in root mean square about their mean; in two planes to nearest up to 2^-17, 2^-19 = 19e-7 in root mean
square.  KAPPA is 4e-7, and OUT |out| at most 2^-16 0.05 |S| = 8e-7 |S| where |out| <= |S| / 20: that is for tokens that see more
than a few slots, of which the last, with an odd number of them, has no partner.
"""
import torch

from synth.configs import BF16, F32
from tests.kv8_planes import KAPPA, OUT, SIGMA_Q  # noqa: F401
from tests.kv8_planes import errors  # noqa: F401
from tests.kv8_ref import act64, f32, stored
from tests.paged_ref import Pool

MANY = 200   # slots from which on a token's error shows a lost plane

# dtype, q-heads, kv heads, head dim, page, slots of each row: one workgroup a row, shares, both storage types
ATTENTION = [(BF16, 32, 8, 128, 32, [333, 700, 5000]), (BF16, 16, 1, 64, 16, [200, 3000]), (BF16, 4, 2, 128, 64, [20000]), (BF16, 3, 3, 64, 16, [299, 800]),
             (F32, 8, 2, 128, 64, [240, 1500]), (F32, 4, 4, 64, 16, [300])]

# dtype, q-heads, kv heads, head dim, page, (slots held before, tokens) of each row, the kernel: 0 tiles, else (key shares, waves)
PROMPTS = [
    (F32, 8, 2, 128, 16, [(230, 50)], 0), (BF16, 8, 2, 64, 16, [(2000, 9)], 0), (BF16, 32, 8, 128, 32, [(200, 200), (300, 40)], 0),
    (BF16, 32, 8, 64, 32, [(0, 1500)], (2, 8)), (BF16, 32, 8, 128, 32, [(0, 1500)], (2, 8)), (BF16, 16, 1, 128, 16, [(17001, 260)], (2, 8)),
    (BF16, 16, 1, 64, 256, [(9000, 4200)], (1, 4)), (BF16, 16, 1, 128, 32, [(200, 5000)], (1, 4)), (BF16, 32, 8, 128, 32, [(100, 300)] * 20, (1, 4)),
    (BF16, 16, 1, 64, 32, [(9000, 2200)], (1, 8)), (BF16, 16, 1, 128, 64, [(9000, 2200)], (1, 8)), (BF16, 16, 1, 128, 32, [(0, 7000)], (1, 8)),
    # tokens on both sides of 16,384 slots, and behind them, in calls that fill the card
    (BF16, 16, 1, 64, 32, [(15500, 2200)], (1, 8)), (BF16, 16, 1, 128, 64, [(15500, 2200)], (1, 8)), (BF16, 16, 1, 64, 256, [(14000, 4200)], (1, 4)),
    (BF16, 16, 1, 128, 16, [(14000, 4200)], (1, 4)), (BF16, 16, 1, 128, 32, [(17000, 7000)], (1, 8))]


def make(ham, dtype, H, Hk, hd, P, lens, seed=31):
    """Shape, and a pool whose rows hold `lens` slots of pairs in pages of no order, everything else NaN; the generator."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // P) for n in lens]
    s = ham.paged_shape(dtype, len(lens), H, Hk, hd, P, sum(need) + 3, max(need) + 1)
    pool = Pool(s, fill=0xFF)
    ids = torch.randperm(s.n_pages, generator=g).tolist()
    for r, n in enumerate(lens):
        pool.len[r] = n
        pool.table[r][:need[r]] = [ids.pop() for _ in range(need[r])]
        k, v = torch.randn(2, n + n % 2, Hk, hd, generator=g)
        k[1::2] = k[::2] + 0.02 * torch.randn(k[::2].shape, generator=g)
        v[1::2] = -v[::2]
        pool.append(r, 0, *(stored(t.double(), dtype)[:n] for t in (k, v)))
    return s, pool, g


def some_tokens(rows):
    """Of packed rows: (packed row, row, slots that its token sees), the first, last and middle ones and those next to 16,384 slots."""
    out, o = [], 0
    for r, (held, c) in enumerate(rows):
        near = [16384 - held + i for i in (-33, -2, -1, 0, 1, 30, 65)]
        pick = {0, 1, c // 3, c // 2, c - 33, c - 2, c - 1, *near}
        out += [(o + i, r, held + i + 1) for i in sorted(pick) if 0 <= i < c]
        o += c
    return out


def attention(pool, q, seen, planes=None):
    """Rows of q float64 [n][H][hd], of (row, slots seen): outputs and S in float64; with `planes` = (how many, "cut" or "near") the
    outputs with the kernel's roundings, and S."""
    n, H, hd = q.shape
    Hk = pool.s.n_kv_heads
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    for r in sorted({r for r, _ in seen}):
        at = [i for i, (x, _) in enumerate(seen) if x == r]
        last = torch.tensor([seen[i][1] for i in at])
        k, v = pool.keys_values(r, int(last.max()))
        hidden = torch.arange(k.shape[1]) >= last[:, None]
        for h in range(H):
            kh, vh, qh = k[h * Hk // H], v[h * Hk // H], q[at, h]
            p = torch.softmax((qh @ kh.T / hd ** 0.5).masked_fill(hidden, -float("inf")), -1)
            spread[at, h] = (p.square() @ vh.square()).sqrt()
            if planes is None:
                out[at, h] = p @ vh
                continue
            sc = torch.zeros(len(at), kh.shape[0], dtype=torch.float64)
            for i in range(0, hd, 16):
                sc = f32(sc + qh[:, i:i + 16] @ kh[:, i:i + 16].T)
            sc = f32(sc * f32(torch.tensor(1.4426950408889634 / hd ** 0.5, dtype=torch.float64)))
            sc = sc.masked_fill(hidden, -float("inf"))
            p = f32(torch.exp2(f32(sc - sc.amax(-1, keepdim=True))))
            out[at, h] = f32(f32(cut(p, *planes) @ vh) / f32(p.sum(-1, keepdim=True)))
    if planes is not None:
        out = act64(out.reshape(n, H * hd), pool.s.dtype)
        out = (out if pool.s.dtype == F32 else out[:, :H * hd] + out[:, H * hd:]).view(n, H, hd)
    return out, spread


def cut(p, n, how):
    """The sum of n bf16 planes of fp32 values (all of it with n = 0)."""
    if n == 0:
        return p
    x, total = p.float(), torch.zeros_like(p)
    for _ in range(n):
        hi = x.bfloat16().float() if how == "near" else (x.view(torch.int32) & -65536).view(torch.float32)
        total += hi.double()
        x = x - hi
    return total
