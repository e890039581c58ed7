"""Timed cases of the operators on a KV cache in 8 bits (``ham_op_kv8_*``), beside their plain forms.

Per (row, kv head) such a cache holds closed blocks of 32 slots, K and V as e4m3 codes with one fp32 scale each and the
least and greatest code of K per channel, and one open block in the storage type (the slots past the last full block).
Kinds of case, by the entry point that a pass calls:

* ``append``  RoPE of projection rows and the append of their K and V: single tokens and prompts
              (``ham_op_kv8_append``)
* ``pack``    a filled cache in the storage type, as a prefill leaves it, into 8 bits (``ham_op_kv8_pack``)
* ``attn``    attention of one query row per sequence over every slot (``ham_op_kv8_attention``)
* ``sparse``  the same over listed blocks and the open one
* ``select``  the list: the blocks whose keys' upper bounds of q . k are greatest (``ham_op_kv8_select``)

The plain forms are elementary torch operations in 32 bits; the block scores and their order are taken in 64, since the
choice lies next to a border.  ``exact`` computes the same in float64, rounding where the definition rounds to a stored
type.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32  # slots
F8 = torch.float8_e4m3fn
F8_MAX = 448.0


def listed():
    def case(name, kind, rows, hd, kv, **kw):
        return dict({"name": name, "kind": kind, "dtype": "bf16", "rows": rows, "H": 32, "Hk": 8, "hd": hd, "kv": kv,
                     "tokens": 0, "n": 0}, **kw)

    return [
        # one token of one sequence, 1B shape: the smallest write, latency
        case("append_1b_b1", "append", 1, 64, 700, tokens=1),
        # one token of each sequence of a full batch, 8B shape; some rows close a block
        case("append_8b_b32", "append", 32, 128, 2048, tokens=1),
        # prompts of odd lengths that continue a chat of odd length, 8B shape
        case("append_8b_prompts", "append", 4, 128, 333, tokens=4001),
        # a prompt of the tiny fp32 model
        case("append_tiny_f32", "append", 1, 64, 0, tokens=64, dtype="f32", H=4, Hk=2),
        # what a prefill of four long prompts leaves in one layer
        case("pack_8b_4x8190", "pack", 4, 128, 8190),
        # decode attention of a single sequence, 1B shape: launches and latency
        case("attn_1b_b1", "attn", 1, 64, 700),
        # ... of a full ragged batch, 8B shape
        case("attn_8b_b32", "attn", 32, 128, 2560),
        # ... of few long contexts, 8B shape: the largest call
        case("attn_8b_long", "attn", 4, 128, 33300),
        # ... of fp32 activations and many queries to a kv head
        case("attn_f32_group8", "attn", 2, 64, 5003, dtype="f32", H=32, Hk=4),
        # the long contexts again, 64 blocks (2,048 slots) of each kv head
        case("sparse_8b_long", "sparse", 4, 128, 33300, n=64),
        # the choice of those blocks
        case("select_8b_long", "select", 4, 128, 33300, n=64),
        # the choice in a full batch
        case("select_8b_b32", "select", 32, 128, 2560, n=16),
    ]


def draw(rng):
    def spread(lo, hi):  # over the logarithm, odd sizes among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("append", "append", "pack", "attn", "attn", "attn", "sparse", "select"))
    H, Hk = rng.choice(((32, 8), (32, 8), (4, 2), (8, 8), (9, 3), (32, 4), (16, 1)))
    rows = spread(1, 64)
    c = {"kind": kind, "dtype": "f32" if rng.random() < 0.2 else "bf16", "rows": rows, "H": H, "Hk": Hk,
         "hd": rng.choice((64, 128)), "kv": spread(1, min(33000, 130000 // rows)), "tokens": 0, "n": 0}
    if kind == "append":
        if rng.random() < 0.5:
            c.update(tokens=1, kv=spread(1, min(33000, 65000 // rows)))
        else:
            c.update(tokens=spread(2, 16000 // rows), kv=spread(1, 2000))
    elif kind == "pack":
        c["kv"] = spread(1, min(33000, 32000 // rows))
    elif kind in ("sparse", "select"):
        c["kv"] = spread(200, max(201, min(33000, 130000 // rows)))
        c["n"] = spread(1, max(2, c["kv"] // (2 * BLOCK)))
    return c


# ---------------------------------------------------------------- the cache buffer
def _storage(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _blocks(case):
    return (case["kv"] + case["tokens"] + 63) // 64 * 2


def _regions(case, cache):
    """The regions of a cache buffer (ham_op_kv8_info), each aligned to 256 bytes."""
    R, Hk, NB, hd, t = case["rows"], case["Hk"], _blocks(case), case["hd"], _storage(case)
    out, at = {}, 0
    for name, shape, dt, size in (("codes", (R, Hk, NB, 2, BLOCK * hd), F8, 1), ("scales", (R, Hk, NB, 2), torch.float32, 4),
                                  ("bounds", (R, Hk, NB, hd // 8, 2, 8), F8, 1), ("open", (R, Hk, 2, BLOCK, hd), t, t.itemsize)):
        n = math.prod(shape) * size
        if cache is not None:
            out[name] = cache[at:at + n].view(dt).view(shape)
        at += (n + 255) // 256 * 256
    return out if cache is not None else at


def _to_lanes(k, v):
    """Codes of K and V [..., 32 slots, hd] in the order of the buffer, [..., 32 * hd] each."""
    lead, hd = k.shape[:-2], k.shape[-1]
    n = len(lead)
    k = k.reshape(*lead, 4, 2, 4, hd // 64, 4, 16)      # slot 8a + 4t + b, channel 64i + 16g + e
    k = k.permute(*range(n), n + 1, n + 3, n + 4, n, n + 2, n + 5).reshape(*lead, BLOCK * hd)
    v = v.reshape(*lead, 4, 8, hd // 32, 2, 16)         # slot 8g + e, channel 32p + 16h + r
    v = v.permute(*range(n), n + 2, n, n + 4, n + 3, n + 1).reshape(*lead, BLOCK * hd)
    return k, v


def _from_lanes(k, v, hd):
    """The inverse of _to_lanes."""
    lead = k.shape[:-1]
    n = len(lead)
    k = k.reshape(*lead, 2, hd // 64, 4, 4, 4, 16).permute(*range(n), n + 3, n, n + 4, n + 1, n + 2, n + 5)
    v = v.reshape(*lead, hd // 32, 4, 16, 2, 8).permute(*range(n), n + 1, n + 4, n, n + 3, n + 2)
    return k.reshape(*lead, BLOCK, hd), v.reshape(*lead, BLOCK, hd)


def _coded(x):
    """Blocks [..., 32, hd] of fp32 values that the storage type holds -> codes as fp32, scales [...]."""
    top = x.abs().amax((-1, -2))
    scale = top / torch.full_like(top, F8_MAX)   # by a tensor: a division by a number may multiply by its inverse
    inv = torch.where(scale >= torch.finfo(torch.float32).tiny, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    return (x * inv[..., None, None]).clamp(-F8_MAX, F8_MAX).to(F8).float(), scale


def _close(reg, r, h, b, k, v):
    """Writes the full blocks k, v [n, 32, hd] (fp32 values of the storage type) as blocks b of kv heads h of rows r."""
    ck, sk = _coded(k)
    cv, sv = _coded(v)
    reg["codes"].view(torch.uint8)[r, h, b] = torch.stack(_to_lanes(ck, cv), 1).to(F8).view(torch.uint8)
    reg["scales"][r, h, b] = torch.stack([sk, sv], 1)
    least = torch.stack([ck.amin(1), ck.amax(1)], 1).view(-1, 2, k.shape[-1] // 8, 8).transpose(1, 2)
    reg["bounds"].view(torch.uint8)[r, h, b] = least.to(F8).view(torch.uint8)


# ---------------------------------------------------------------- inputs
def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 2 + 1)


def _act(x, case):
    """fp32 rows in the activation layout: as they are, or bf16 hi and lo planes."""
    if case["dtype"] == "f32":
        return x.contiguous()
    hi = x.to(torch.bfloat16)
    return torch.cat([hi, (x - hi.float()).to(torch.bfloat16)], -1)


def _from_act(x, case):
    if case["dtype"] == "f32":
        return x
    W = x.shape[-1] // 2
    return x[..., :W].float() + x[..., W:].float()


def _keys_values(case, g, rows, slots, kv_heads):
    """K and V of a context: channels of unequal size and mean, keys that drift from block to block."""
    hd = case["hd"]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    size = torch.exp(0.5 * randn(kv_heads, 1, 1, hd))
    K = randn(rows, kv_heads, slots // BLOCK, BLOCK, hd) + randn(rows, kv_heads, slots // BLOCK, 1, hd) + randn(kv_heads, 1, 1, hd)
    V = randn(rows, kv_heads, slots // BLOCK, BLOCK, hd)
    t = _storage(case)
    return K.mul_(0.6 * size).to(t), V.to(t)


def _lengths(case, g, longest):
    """Ragged: between four fifths of the longest and the longest, one row at it."""
    n = torch.randint(longest - longest // 5, longest + 1, (case["rows"],), generator=g, device=DEV, dtype=torch.int32)
    n[0] = longest
    return n


def prepare(case, seed):
    g = _rng(seed)
    R, H, Hk, hd, NB, T = case["rows"], case["H"], case["Hk"], case["hd"], _blocks(case), case["tokens"]
    s = {"case": case, "n": _lengths(case, g, case["kv"]), "err": torch.zeros(R, dtype=torch.int32, device=DEV),
         "cache": torch.zeros(_regions(case, None), dtype=torch.uint8, device=DEV), "on": torch.ones(R, dtype=torch.int32, device=DEV),
         "ws": torch.zeros(_workspace_bytes(case), dtype=torch.uint8, device=DEV)}
    reg = s["reg"] = _regions(case, s["cache"])
    K, V = _keys_values(case, g, R, NB * BLOCK, Hk)
    if case["kind"] == "pack":
        s["K"] = K.view(R, Hk, NB * BLOCK, hd)
        s["VT"] = V.transpose(3, 4).contiguous()
        return s
    # the cache of the slots held: closed blocks, and the open block of each row
    ck, sk = _coded(K.float())
    cv, sv = _coded(V.float())
    reg["codes"].copy_(torch.stack(_to_lanes(ck, cv), 3))
    reg["scales"].copy_(torch.stack([sk, sv], 3))
    reg["bounds"].copy_(torch.stack([ck.amin(3), ck.amax(3)], 3).view(R, Hk, NB, 2, hd // 8, 8).transpose(3, 4))
    del ck, cv
    at = (s["n"].long() // BLOCK).clamp(max=NB - 1)
    row = torch.arange(R, device=DEV)
    reg["open"].copy_(torch.stack([K[row, :, at], V[row, :, at]], 2))
    del K, V
    if case["kind"] == "append":
        s["qkv"] = torch.randn(R, T, (H + 2 * Hk) * hd, generator=g, device=DEV)
        pos = s["n"][:, None] + torch.arange(T, device=DEV)
        angle = pos[..., None].double() * 500000.0 ** (-2.0 * torch.arange(hd // 2, device=DEV).double() / hd)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["count"] = _lengths(case, g, T)
        s["q"] = torch.zeros(R, T, H * hd * (1 if case["dtype"] == "f32" else 2), dtype=_storage(case), device=DEV)
        return s
    s["q"] = _act(1.5 * torch.randn(R, H * hd, generator=g, device=DEV), case)
    if case["kind"] == "select":
        s["blocks"] = torch.zeros(R, Hk, case["n"], dtype=torch.int32, device=DEV)
        s["n_blocks"] = torch.zeros(R, Hk, dtype=torch.int32, device=DEV)
        return s
    s["out"] = torch.zeros_like(s["q"])
    if case["kind"] == "sparse":
        # a list of n blocks of each kv head, ascending, as the choice leaves it (fewer where a row has fewer)
        closed = (s["n"].long() // BLOCK)[:, None]
        u = torch.rand(R, Hk, NB, generator=g, device=DEV)
        u = torch.where(torch.arange(NB, device=DEV) < closed[..., None], u, torch.full_like(u, 2.0))
        u, i = u.sort(-1)
        i = torch.where(u < 2.0, i, torch.full_like(i, NB))[..., :case["n"]].sort(-1).values
        i = torch.nn.functional.pad(i, (0, case["n"] - i.shape[-1]), value=NB)
        s["blocks"] = torch.where(i < NB, i, torch.full_like(i, -1)).to(torch.int32).contiguous()
        s["n_blocks"] = (i < NB).sum(-1).to(torch.int32)
    return s


def _workspace_bytes(case):
    """What a caller keeps for the kernels' intermediate records: at least ham_op_kv8_workspace_bytes."""
    pairs, grp = case["rows"] * case["Hk"], case["H"] // case["Hk"]
    return max((pairs + 2048) * grp * (case["hd"] + 2) * 4, pairs * _blocks(case) * 4) + 4096


# ---------------------------------------------------------------- one pass, plain
def _rope(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_append(s):
    case, reg = s["case"], s["reg"]
    R, H, Hk, hd, T = case["rows"], case["H"], case["Hk"], case["hd"], case["tokens"]
    x = s["qkv"].view(R, T, H + 2 * Hk, hd)
    cos, sin = s["cos"][:, :, None], s["sin"][:, :, None]
    new = torch.arange(T, device=DEV) < s["count"][:, None]
    q = _act(_rope(x[:, :, :H], cos, sin).view(R, T, H * hd), case)
    s["q"].copy_(torch.where(new[..., None], q, s["q"]))
    t = _storage(case)
    # the slots from the start of each row's first touched block on: old ones, then new ones
    W = (T + BLOCK - 1) // BLOCK * BLOCK + BLOCK
    first, off = s["n"].long() // BLOCK, s["n"].long() % BLOCK
    w = torch.arange(W, device=DEV)
    src = w - off[:, None]
    end = off + s["count"]
    kv = torch.stack([_rope(x[:, :, H:H + Hk], cos, sin), x[:, :, H + Hk:]], 2).to(t)          # [R][T][2][Hk][hd]
    kv = kv.gather(1, src.clamp(0, T - 1)[:, :, None, None, None].expand(R, W, 2, Hk, hd))
    kv = kv.permute(0, 3, 2, 1, 4)                                                             # [R][Hk][2][W][hd]
    old = torch.nn.functional.pad(reg["open"], (0, 0, 0, W - BLOCK))
    kv = torch.where((src >= 0)[:, None, None, :, None], kv, old)
    blocks = kv.float().view(R, Hk, 2, W // BLOCK, BLOCK, hd)
    full = (torch.arange(W // BLOCK, device=DEV) + 1) * BLOCK <= end[:, None]
    r, b = full.nonzero(as_tuple=True)
    h = torch.arange(Hk, device=DEV).repeat(r.numel())
    r, b = r.repeat_interleave(Hk), b.repeat_interleave(Hk)
    _close(reg, r, h, first[r] + b, blocks[r, h, 0, b], blocks[r, h, 1, b])
    # the open block: the slots past the last full one
    last = end // BLOCK
    lane = torch.arange(BLOCK, device=DEV)
    at = (last[:, None] * BLOCK + lane).clamp(max=W - 1)
    tail = kv.gather(3, at[:, None, None, :, None].expand(R, Hk, 2, BLOCK, hd))
    keep = lane < (end % BLOCK)[:, None]
    reg["open"].copy_(torch.where(keep[:, None, None, :, None], tail, reg["open"]))
    return {"q": s["q"], "codes": reg["codes"], "scales": reg["scales"], "bounds": reg["bounds"], "open": reg["open"], "err": s["err"]}


def _plain_pack(s):
    case, reg = s["case"], s["reg"]
    R, Hk, hd, NB = case["rows"], case["Hk"], case["hd"], _blocks(case)
    K = s["K"].float().view(R, Hk, NB, BLOCK, hd)
    V = s["VT"].float().transpose(3, 4)
    closed = s["n"].long() // BLOCK
    r, h, b = (torch.arange(NB, device=DEV) < closed[:, None, None]).expand(R, Hk, NB).nonzero(as_tuple=True)
    _close(reg, r, h, b, K[r, h, b], V[r, h, b])
    row = torch.arange(R, device=DEV)
    at = closed.clamp(max=NB - 1)
    tail = torch.stack([K[row, :, at], V[row, :, at]], 2).to(_storage(case))
    keep = torch.arange(BLOCK, device=DEV) < (s["n"] % BLOCK)[:, None]
    reg["open"].copy_(torch.where(keep[:, None, None, :, None], tail, reg["open"]))
    return {"codes": reg["codes"], "scales": reg["scales"], "bounds": reg["bounds"], "open": reg["open"], "err": s["err"]}


def _plain_attention(s):
    case, reg = s["case"], s["reg"]
    R, H, Hk, hd, NB = case["rows"], case["H"], case["Hk"], case["hd"], _blocks(case)
    q = _from_act(s["q"], case).view(R, Hk, H // Hk, hd) / math.sqrt(hd)
    c = reg["codes"].float()
    K, V = _from_lanes(c[:, :, :, 0], c[:, :, :, 1], hd)
    K = (K * reg["scales"][..., 0, None, None]).view(R, Hk, NB * BLOCK, hd)
    V = (V * reg["scales"][..., 1, None, None]).view(R, Hk, NB * BLOCK, hd)
    K = torch.cat([K, reg["open"][:, :, 0].float()], 2)
    V = torch.cat([V, reg["open"][:, :, 1].float()], 2)
    block = torch.arange(NB, device=DEV)
    seen = (block < (s["n"] // BLOCK)[:, None, None]).expand(R, Hk, NB)
    if "blocks" in s:
        on = torch.zeros(R, Hk, NB + 1, dtype=torch.bool, device=DEV)
        on.scatter_(2, torch.where(s["blocks"] < 0, torch.full_like(s["blocks"], NB), s["blocks"]).long(), True)
        seen = seen & on[..., :NB]
    rest = torch.arange(BLOCK, device=DEV) < (s["n"] % BLOCK)[:, None, None]
    seen = torch.cat([seen.repeat_interleave(BLOCK, 2), rest.expand(R, Hk, BLOCK)], 2)[:, :, None]
    sc = (q @ K.transpose(2, 3)).masked_fill(~seen, -math.inf)
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    o = (p @ V) / p.sum(-1, keepdim=True)
    s["out"].copy_(_act(o.view(R, H * hd), case))
    return {"out": s["out"], "err": s["err"]}


def _plain_select(s):
    case, reg = s["case"], s["reg"]
    R, H, Hk, hd, NB, n = case["rows"], case["H"], case["Hk"], case["hd"], _blocks(case), case["n"]
    q = _from_act(s["q"], case).view(R, Hk, H // Hk, hd).double()
    b = reg["bounds"].double()
    lo, hi = b[..., 0, :].reshape(R, Hk, NB, hd), b[..., 1, :].reshape(R, Hk, NB, hd)
    top = hi @ q.clamp(min=0).transpose(2, 3).contiguous() + lo @ q.clamp(max=0).transpose(2, 3).contiguous()
    score = (top.amax(-1) * reg["scales"][..., 0].double()).float()
    closed = (s["n"].long() // BLOCK)[:, None]
    there = torch.arange(NB, device=DEV) < closed[..., None]
    score = score.masked_fill(~there, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :n]   # equal scores: the lowest index first
    best = torch.nn.functional.pad(best, (0, n - best.shape[-1]), value=NB)
    best = torch.where(best < closed[..., None], best, torch.full_like(best, NB)).sort(-1).values
    s["blocks"].copy_(torch.where(best < NB, best, torch.full_like(best, -1)))
    s["n_blocks"].copy_((best < NB).sum(-1))
    return {"blocks": s["blocks"], "n_blocks": s["n_blocks"], "err": s["err"]}


def _kernels(s):
    from paper_2505_20438_amd import ham
    case, reg = s["case"], s["reg"]
    shape = ham.kv8_shape(ham.HAM_F32 if case["dtype"] == "f32" else ham.HAM_BF16, case["rows"], case["H"], case["Hk"],
                          case["hd"], _blocks(case) * BLOCK)
    stream = torch.cuda.current_stream().cuda_stream
    if case["kind"] == "append":
        ham.ham_op_kv8_append(shape, s["qkv"], s["cos"], s["sin"], s["n"], s["count"], s["cache"], s["q"], s["err"], stream)
        return {"q": s["q"], "codes": reg["codes"], "scales": reg["scales"], "bounds": reg["bounds"], "open": reg["open"], "err": s["err"]}
    if case["kind"] == "pack":
        ham.ham_op_kv8_pack(shape, s["K"], s["VT"], s["n"], case["kv"], s["cache"], s["err"], stream)
        return {"codes": reg["codes"], "scales": reg["scales"], "bounds": reg["bounds"], "open": reg["open"], "err": s["err"]}
    if case["kind"] == "select":
        ham.ham_op_kv8_select(shape, s["q"], s["cache"], s["n"], s["on"], case["kv"], case["n"], 0, 0, s["blocks"], s["n_blocks"],
                              s["err"], s["ws"], stream)
        return {"blocks": s["blocks"], "n_blocks": s["n_blocks"], "err": s["err"]}
    ham.ham_op_kv8_attention(shape, s["q"], s["cache"], s["n"], s["on"], case["kv"], s.get("blocks"), s.get("n_blocks"), s["out"],
                             s["err"], s["ws"], stream)
    return {"out": s["out"], "err": s["err"]}


def run(state):
    if own:
        return _kernels(state)
    return {"append": _plain_append, "pack": _plain_pack, "attn": _plain_attention, "sparse": _plain_attention,
            "select": _plain_select}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- work
def work(case):
    R, H, Hk, hd, kv, T = case["rows"], case["H"], case["Hk"], case["hd"], case["kv"], case["tokens"]
    es = 4 if case["dtype"] == "f32" else 2
    slot = 2 * hd + (2 * hd + 8) / BLOCK      # codes of K and V, bounds and scales, of a slot in a closed block
    if case["kind"] == "append":
        n = R * (T * 0.9 if T > 1 else 1)
        out = slot if T > 1 else 2 * hd * es  # a single token goes to the open block
        return {"bytes": n * (4 * (H + 2 * Hk) * hd + 4 * hd + 4 * H * hd + Hk * out), "flops": n * 3.0 * (H + Hk) * hd}
    kv = R * (kv * 0.9 if R > 1 else kv)
    if case["kind"] == "pack":
        return {"bytes": kv * Hk * (2 * hd * es + slot), "flops": kv * Hk * 6.0 * hd}
    rows = R * H * hd * 8.0
    if case["kind"] == "select":
        return {"bytes": kv / BLOCK * Hk * (2 * hd + 4) + R * H * hd * 4 + R * Hk * case["n"] * 4, "flops": kv / BLOCK * H * hd * 4}
    if case["kind"] == "sparse":
        kv = min(kv, R * case["n"] * BLOCK)
    return {"bytes": kv * Hk * (2 * hd + 8 / BLOCK) + rows, "flops": 4.0 * kv * H * hd}


# ---------------------------------------------------------------- float64
def _f32(x):
    """float64 values that an fp32 operation of the definition rounds."""
    return x.float().double()


def _stored64(x, case):
    return x.float().to(_storage(case)).double()


def _code_index(hd):
    """Where K and V of (slot, channel) are within the codes of a block."""
    s, d = torch.arange(BLOCK, device=DEV)[:, None], torch.arange(hd, device=DEV)[None]
    k = (((s // 4 % 2) * (hd // 64) + d // 64) * 64 + d // 16 % 4 * 16 + s // 8 * 4 + s % 4) * 16 + d % 16
    v = ((d // 32 * 4 + s // 8) * 16 + d % 16) * 16 + d // 16 % 2 * 8 + s % 8
    return k, v


def _exact_block(x, case):
    """A block [32][hd] of stored values in float64 -> codes, scale."""
    scale = _f32(x.abs().max() / F8_MAX)
    inv = _f32(1.0 / scale) if scale >= 2.0 ** -126 else torch.zeros_like(scale)
    return _f32(x * inv).clamp(-F8_MAX, F8_MAX).float().to(F8).double(), scale


def _exact_write(case, reg, kv, r, start, end):
    """Slots [start, end) of row r from kv [2][end][Hk][hd] in float64; `reg` in float64 too, slots before from its open block."""
    hd, first, last = case["hd"], start // BLOCK, end // BLOCK
    ki, vi = _code_index(hd)
    for h in range(case["Hk"]):
        x = kv[:, :, h].clone()
        x[:, first * BLOCK:start] = reg["open"][r, h, :, :start - first * BLOCK]
        for b in range(first, last):
            for j, at in ((0, ki), (1, vi)):
                c, reg["scales"][r, h, b, j] = _exact_block(x[j, b * BLOCK:(b + 1) * BLOCK], case)
                reg["codes"][r, h, b, j, at.reshape(-1)] = c.reshape(-1)
                if j == 0:
                    d = torch.arange(hd, device=DEV)
                    reg["bounds"][r, h, b, d // 8, 0, d % 8] = c.min(0).values
                    reg["bounds"][r, h, b, d // 8, 1, d % 8] = c.max(0).values
        a = max(start, last * BLOCK)
        reg["open"][r, h, :, a - last * BLOCK:end - last * BLOCK] = x[:, a:end]


def _dequantised(case, reg, r, h):
    """K and V [blocks][32][hd] of a (row, kv head) in float64."""
    ki, vi = _code_index(case["hd"])
    c, sc = reg["codes"][r, h].double(), reg["scales"][r, h].double()
    return c[:, 0][:, ki] * sc[:, 0, None, None], c[:, 1][:, vi] * sc[:, 1, None, None]


def exact(case, seed):
    s = prepare(case, seed)
    reg, R, H, Hk, hd = s["reg"], case["rows"], case["H"], case["Hk"], case["hd"]
    lens = s["n"].tolist()
    if case["kind"] in ("append", "pack"):
        if R * Hk * (case["tokens"] if case["kind"] == "append" else case["kv"]) > 300_000:
            return None  # a block at a time takes too long
        out = {k: reg[k].double() for k in ("codes", "scales", "bounds", "open")}
        if case["kind"] == "pack":
            for r in range(R):
                v = s["VT"][r].double().transpose(2, 3).reshape(Hk, -1, hd)
                kv = torch.stack([s["K"][r].double(), v]).transpose(1, 2)
                _exact_write(case, out, kv[:, :lens[r]], r, 0, lens[r])
            return dict(out, err=None)
        x = s["qkv"].double().view(R, -1, H + 2 * Hk, hd)
        c, sn = s["cos"].double()[:, :, None], s["sin"].double()[:, :, None]
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        rot = torch.cat([_f32(_f32(a * c) - _f32(b * sn)), _f32(_f32(b * c) + _f32(a * sn))], -1)
        out["q"] = s["q"].double()
        for r, n in enumerate(s["count"].tolist()):
            q = rot[r, :n, :H].reshape(n, H * hd)
            if case["dtype"] == "bf16":
                hi = _stored64(q, case)
                q = torch.cat([hi, _stored64(q - hi, case)], -1)
            out["q"][r, :n] = q
            kv = torch.zeros(2, lens[r] + n, Hk, hd, dtype=torch.float64, device=DEV)
            kv[0, lens[r]:], kv[1, lens[r]:] = _stored64(rot[r, :n, H:H + Hk], case), _stored64(x[r, :n, H + Hk:], case)
            _exact_write(case, out, kv, r, lens[r], lens[r] + n)
        return dict(out, err=None)
    if case["kind"] == "select":
        return None  # whole numbers
    q = _from_act(s["q"], case).double().view(R, H, hd)
    o = torch.zeros(R, H, hd, dtype=torch.float64, device=DEV)
    for r in range(R):
        for h in range(Hk):
            K, V = _dequantised(case, reg, r, h)
            at = torch.arange(lens[r] // BLOCK, device=DEV)
            if "blocks" in s:
                at = s["blocks"][r, h, :int(s["n_blocks"][r, h])].long()
            tail = reg["open"][r, h, :, :lens[r] % BLOCK].double()
            K, V = torch.cat([K[at].view(-1, hd), tail[0]]), torch.cat([V[at].view(-1, hd), tail[1]])
            j = slice(h * H // Hk, (h + 1) * H // Hk)
            o[r, j] = torch.softmax(q[r, j] @ K.T / math.sqrt(hd), -1) @ V
    o = o.view(R, H * hd)
    if case["dtype"] == "bf16":
        hi = _stored64(o, case)
        o = torch.cat([hi, _stored64(o - hi, case)], -1)
    return {"out": o, "err": None}
