"""The 8-bit KV cache and the operators over it in float64 on the CPU, from their definition in include/ham_ops.h: rounding
to fp32, the storage type and e4m3 exactly where it says so.

Tolerances.  Cache contents (codes, scales, bounds, open block, rotated q) are rounded step by step by the definition: they
are held to it bit for bit, and so are chosen blocks (scores are fp64 sums; an fp32 rounding of two such sums in different
order can differ only where they straddle a border, at 2^-53 against 2^-24).  Attention: FILLED_TOL of attention_bounds.py, which
a lost or doubled slot exceeds; the terms here are smaller (weights of 24 significant bits, outputs as hi/lo pairs or fp32,
fp32 scores over the head dim).  kv8_planes.py has the bounds that a lost bf16 plane exceeds.
"""
import numpy as np
import torch

from synth.configs import BF16

B = 32
F8 = torch.float8_e4m3fn


def storage(dtype):
    return torch.bfloat16 if dtype == BF16 else torch.float32


def f32(x):
    return x.to(torch.float32).to(torch.float64)


def stored(x, dtype):
    """float64 -> float64 of the storage type (through fp32)."""
    return x.to(torch.float32).to(storage(dtype)).to(torch.float64)


def code_index(hd):
    """Byte of (slot, channel) in the K codes and in the V codes of a block, by the header's formulas."""
    s, d = np.meshgrid(np.arange(B), np.arange(hd), indexing="ij")
    k = ((s // 4 % 2 * (hd // 64) + d // 64) * 64 + d // 16 % 4 * 16 + s // 8 * 4 + s % 4) * 16 + d % 16
    v = ((d // 32 * 4 + s // 8) * 16 + d % 16) * 16 + d // 16 % 2 * 8 + s % 8
    return torch.from_numpy(k), torch.from_numpy(v)


def quantise(x):
    """Blocks [..., 32, hd] of stored values -> codes (float8), scales (fp32)."""
    top = x.abs().amax((-1, -2))
    scale = f32(top / 448.0)
    inv = torch.where(scale >= 2.0 ** -126, f32(1.0 / scale), torch.zeros_like(scale))
    y = f32(x * inv[..., None, None])
    y = torch.where(torch.isnan(y), torch.full_like(y, -448.0), y).clamp(-448.0, 448.0)
    bad = ~torch.isfinite(top)
    return y.to(torch.float32).to(F8), torch.where(bad, torch.full_like(scale, float("nan")), scale).to(torch.float32)


class Cache:
    """A cache buffer on the CPU, bytes and regions (typed views of it)."""

    def __init__(self, shape, info, nbytes, fill=None):
        self.shape = shape
        self.buf = torch.full((nbytes,), 0xAB, dtype=torch.uint8) if fill is None else fill
        R, Hk, NB, hd = shape.rows, shape.n_kv_heads, shape.slots_cap // B, shape.head_dim
        t = storage(shape.dtype)

        def view(off, dt, *dims):
            n = int(np.prod(dims)) * torch.empty(0, dtype=dt).element_size()
            return self.buf[off:off + n].view(dt).view(*dims)
        self.codes = view(info["codes"], torch.uint8, R, Hk, NB, 2, B * hd)
        self.scales = view(info["scales"], torch.float32, R, Hk, NB, 2)
        self.bounds = view(info["bounds"], torch.uint8, R, Hk, NB, hd // 8, 2, 8)
        self.open = view(info["open"], t, R, Hk, 2, B, hd)
        self.ki, self.vi = code_index(hd)

    def close(self, r, h, b, k, v):
        """Writes block b of (row, kv head) from stored values k, v [32][hd] (float64)."""
        (ck, sk), (cv, sv) = quantise(k), quantise(v)
        self.codes[r, h, b, 0, self.ki.reshape(-1)] = ck.view(torch.uint8).reshape(-1)
        self.codes[r, h, b, 1, self.vi.reshape(-1)] = cv.view(torch.uint8).reshape(-1)
        self.scales[r, h, b, 0], self.scales[r, h, b, 1] = sk, sv
        hd = k.shape[1]
        least = ck.float().amin(0).to(F8).view(torch.uint8).view(hd // 8, 8)
        most = ck.float().amax(0).to(F8).view(torch.uint8).view(hd // 8, 8)
        self.bounds[r, h, b] = torch.stack([least, most], 1)

    def append(self, r, start, k, v):
        """Slots start.. of row r from stored values k, v [n][Hk][hd] (float64)."""
        n, end = k.shape[0], start + k.shape[0]
        if n == 0:
            return
        first, last = start // B, end // B
        for h in range(k.shape[1]):
            x = torch.zeros(2, end - first * B, k.shape[2], dtype=torch.float64)
            off = start - first * B
            x[:, :off] = self.open[r, h, :, :off].double()
            x[0, off:], x[1, off:] = k[:, h], v[:, h]
            for b in range(first, last):
                s = (b - first) * B
                self.close(r, h, b, x[0, s:s + B], x[1, s:s + B])
            a = max(start, last * B)
            self.open[r, h, :, a - last * B:end - last * B] = x[:, a - first * B:].to(self.open.dtype)

    def keys_values(self, r, h, n, blocks=None):
        """What slots < n of (row, kv head) stand for, float64 [slots][hd] each: all closed blocks or those listed, then open."""
        at = torch.arange(n // B) if blocks is None else torch.as_tensor(blocks, dtype=torch.long)
        c, hd = self.codes[r, h, at].view(F8).double(), self.ki.shape[1]
        sc = self.scales[r, h, at].double()
        k = (c[:, 0][:, self.ki] * sc[:, 0, None, None]).reshape(-1, hd)
        v = (c[:, 1][:, self.vi] * sc[:, 1, None, None]).reshape(-1, hd)
        tail = self.open[r, h, :, :n % B].double()
        return torch.cat([k, tail[0]]), torch.cat([v, tail[1]])

    def attention(self, q, lens, lists=None):
        """q [R][H][hd] float64 -> [R][H][hd]; rows without slots are zero."""
        R, H, hd = q.shape
        Hk = self.codes.shape[1]
        out = torch.zeros_like(q)
        for r in range(R):
            for h in range(Hk):
                k, v = self.keys_values(r, h, lens[r], None if lists is None else lists[r][h])
                if k.shape[0]:
                    j = slice(h * H // Hk, (h + 1) * H // Hk)
                    out[r, j] = torch.softmax(q[r, j] @ k.T / hd ** 0.5, -1) @ v
        return out

    def scores(self, q, r, h, n):
        """fp32 scores of the closed blocks of (row, kv head)."""
        H, Hk, hd = q.shape[1], self.codes.shape[1], q.shape[2]
        b = self.bounds[r, h, :n // B].view(F8).double()
        lo, hi = b[:, :, 0].reshape(-1, 1, hd), b[:, :, 1].reshape(-1, 1, hd)
        qs = q[r, h * H // Hk:(h + 1) * H // Hk]
        top = torch.maximum(qs * lo, qs * hi).sum(-1).amax(1) if n // B else torch.zeros(0, dtype=torch.float64)
        s = self.scales[r, h, :n // B].double()
        return (top * torch.where(torch.isnan(s[:, 1]), s[:, 1], s[:, 0])).float()

    def select(self, q, r, h, n, n_blocks, first=0, last=0):
        s = self.scores(q, r, h, n).double()
        s = torch.where(torch.isnan(s), torch.full_like(s, float("inf")), s) + 0.0
        nb = n // B
        always = [b for b in range(nb) if b < first or b >= nb - last]
        if nb <= n_blocks:
            return list(range(nb))
        rest = sorted((b for b in range(nb) if b not in set(always)), key=lambda b: (-float(s[b]), b))
        return sorted(always + rest[:n_blocks - len(always)])


def rope64(x, cos, sin):
    """Rotate-half RoPE with fp32 rounding of each product and sum: x [..., hd], cos, sin [..., hd/2], float64."""
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([f32(f32(a * cos) - f32(b * sin)), f32(f32(b * cos) + f32(a * sin))], -1)


def act64(x, dtype):
    """Rows in the activation layout as the library writes them, float64: fp32, or bf16 hi and lo planes."""
    if dtype != BF16:
        return f32(x)
    hi = stored(x, dtype)
    return torch.cat([hi, stored(x - hi, dtype)], -1)
