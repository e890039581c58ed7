"""The bf16 planes of the attention over an 8-bit cache: inputs on which a lost plane shows, the bound that results are held to,
and the kernel's roundings in float64 with planes to leave out.

The matrix products take bf16 operands.  Codes are exact in bf16; queries are the two planes of a bf16 model's activations or
three planes of an fp32 value, weights (times V's scale) three planes, 24 significant bits.  A plane less leaves 16: two roundings
to nearest, each at most 2^-8 of what it rounds, leave up to 2^-16 of the value and about 2^-19 in root mean square.

Bound of one (row, q-head), 2-norms over the head's channels: KAPPA |S| + OUT |out|, where S is what independent errors of the
weights add up to, S_d^2 = sum_j (p_j v_jd)^2 with p normalised, and OUT the rounding of the output (a bf16 pair: 2^-8 of the low
plane, which is at most 2^-8 of the value; fp32: the sums and the division, a few of 2^-24).  KAPPA is the relative error of a
weight, in root mean square and doubled.  Queries of standard deviation SIGMA_Q = 1/2 give scores of about 1/2 and partial
sums below 1, rounded at 2^-25, at most 96 times (2 or 3 planes of up to 128 channels, sums of 4 products): sqrt(96 / 3) 2^-25 =
1.7e-7.  The score less the maximum, up to 4 in base 2: ln 2 2^-23 / sqrt(3) = 0.5e-7; the power, at 2^-23: 0.7e-7; times V's
scale: 0.3e-7.  Together 1.9e-7.  A lost plane of the weights adds about 2^-19 = 19e-7 |S|, one of an fp32 query half
of that (SIGMA_Q), as it is an error of the scores.

In the inputs with pairs slot 2 i + 1 has the value of slot 2 i with the sign turned, and nearly its key: the two all but cancel,
so that |out| is a small part of |S| and the rounding of a bf16 model's output does not hide the weights'.  (Errors of the
queries cancel with them: those are for the inputs without pairs.)
"""
import torch

from synth.configs import BF16
from tests import kv8_ref
from tests.gpu_util import act_rows, from_act
from tests.kv8_ref import B, Cache, stored

SIGMA_Q = 0.5
KAPPA = 4e-7
OUT = {BF16: 2.0 ** -16, 0: 2.0 ** -22}


def inputs(ham, dtype, H, Hk, hd, lens, pairs, seed=31):
    """Shape, reference cache and act rows of queries (CPU), and the queries in float64 [R][H][hd]."""
    R = len(lens)
    s = ham.kv8_shape(dtype, R, H, Hk, hd, (max(lens) // B + 1) * B)
    n = ham.ham_op_kv8_cache_bytes(s)
    ref = Cache(s, ham.ham_op_kv8_info(s), n, torch.full((n,), 0xFF, dtype=torch.uint8))
    g = torch.Generator().manual_seed(seed)
    for r, slots in enumerate(lens):
        k, v = torch.randn(2, Hk, slots + slots % 2, hd, generator=g)
        if pairs:
            k[:, 1::2] = k[:, ::2] + 0.02 * torch.randn(k[:, ::2].shape, generator=g)
            v[:, 1::2] = -v[:, ::2]
        k, v = (stored(t.double(), dtype)[:, :slots].transpose(0, 1) for t in (k, v))
        ref.append(r, 0, k, v)
    q = act_rows(torch, SIGMA_Q * torch.randn(R, H * hd, generator=g), dtype)
    return s, ref, q, from_act(torch, q, H * hd, dtype).double().view(R, H, hd)


def expected(ref, q, lens, lists=None):
    """Attention and S, float64 [R][H][hd]."""
    R, H, hd = q.shape
    Hk = ref.codes.shape[1]
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    for r in range(R):
        for h in range(H):
            k, v = ref.keys_values(r, h * Hk // H, lens[r], None if lists is None else lists[r][h * Hk // H])
            p = torch.softmax(k @ q[r, h] / hd ** 0.5, 0)
            out[r, h], spread[r, h] = p @ v, (p.square() @ v.square()).sqrt()
    return out, spread


def errors(got, out, spread, dtype):
    """Error of each (row, q-head) as a part of its bound."""
    return (got - out).norm(dim=-1) / (KAPPA * spread.norm(dim=-1) + OUT[dtype] * out.norm(dim=-1))


def planes(x, n):
    """The sum of the first n bf16 planes of fp32 values."""
    x, total = x.float(), torch.zeros_like(x, dtype=torch.float64)
    for _ in range(n):
        p = x.to(torch.bfloat16).float()
        total += p.double()
        x = x - p
    return total


def emulated(ref, q, lens, dtype, q_planes=3, p_planes=3):
    """The attention over every slot with the kernel's roundings: fp32 scores of 32 channels at a time, weights in fp32, then in
    planes; the open block in fp32; the output as it is stored."""
    R, H, hd = q.shape
    Hk = ref.codes.shape[1]
    out = torch.zeros_like(q)
    f32 = kv8_ref.f32
    scale = f32(torch.tensor(1.4426950408889634 / hd ** 0.5, dtype=torch.float64))
    for r in range(R):
        for h in range(H):
            kv, nb = h * Hk // H, lens[r] // B
            c = ref.codes[r, kv, :nb].view(kv8_ref.F8).double()
            kc, vc = c[:, 0][:, ref.ki], c[:, 1][:, ref.vi]
            ks, vs = ref.scales[r, kv, :nb].double().unbind(-1)
            qp = planes(q[r, h], q_planes)
            sc = torch.zeros(nb, B, dtype=torch.float64)
            for i in range(0, hd, 32):
                sc = f32(sc + kc[..., i:i + 32] @ qp[i:i + 32])
            sc = f32(sc * f32(ks * scale)[:, None])
            tail = ref.open[r, kv, :, :lens[r] % B].double()
            st = f32(f32(tail[0] @ q[r, h]) * scale)
            m = torch.cat([sc.reshape(-1), st]).max()
            p, pt = f32(torch.exp2(f32(sc - m))), f32(torch.exp2(f32(st - m)))
            o = (planes(f32(p * vs[:, None]), p_planes)[..., None] * vc).sum((0, 1)) + pt @ tail[1]
            out[r, h] = f32(f32(o) / f32(p.sum() + pt.sum()))
    x = act_rows(torch, out.reshape(R, H * hd).float(), dtype)
    return from_act(torch, x, H * hd, dtype).double().view(R, H, hd)
