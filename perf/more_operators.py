"""Timed cases of the operators on a paged KV cache (``ham_op_paged_*``), beside their plain forms.

A layer's pool holds pages of ``page_slots`` slots of every kv head, K and V in the storage type; row r's slot s lies in page
``table[r][s // page_slots]`` (K of 16 slots in the order of the matrix cores' rows), and ``refs`` counts the rows that hold a
page.  Kinds of case, by the entry point that a pass calls:

* ``append``   RoPE of packed projection rows of sequences of different lengths, K and V into pages (``ham_op_paged_append``)
* ``attn``     attention of one query row per sequence over its pages (``ham_op_paged_attention``)
* ``prompt``   causal attention of packed prompts over their pages, what they held before included (``ham_op_paged_prompt``)
* ``advance``  rows take over other rows' pages, free theirs, and get pages for new slots; a page that two rows share is
               copied before one writes to it (``ham_op_paged_advance``)
* ``compact``  the pages in use move to the front of the pool (``ham_op_paged_compact``)

The plain forms are elementary torch operations in 32 bits, over sequences padded to the longest.  ``exact`` computes the same
in float64, sequence by sequence, rounding where the definition rounds to a stored type.
"""
import math

import torch

own = False

DEV = "cuda:0"


def listed():
    def case(name, kind, rows, hd, kv, **kw):
        return dict({"name": name, "kind": kind, "dtype": "bf16", "rows": rows, "H": 32, "Hk": 8, "hd": hd, "page": 32, "kv": kv,
                     "tokens": 0, "layers": 1, "beams": 0}, **kw)

    return [
        # the prompt of the tiny fp32 model: the smallest write, latency
        case("append_tiny_f32", "append", 1, 64, 0, tokens=64, dtype="f32", H=4, Hk=2, page=16),
        # prompts of 500 to 4,001 tokens that continue chats of up to 333 slots, 8B shape
        case("append_8b_packed", "append", 9, 128, 333, tokens=4001),
        # decode attention of a single sequence, 1B shape: launches and latency
        case("attn_1b_b1", "attn", 1, 64, 700),
        # ... of a full ragged batch, 8B shape
        case("attn_8b_b32", "attn", 32, 128, 2560, page=16),
        # ... of few long contexts, 8B shape
        case("attn_8b_long", "attn", 4, 128, 33300, page=64),
        # one prompt of the 1B shape from its first token
        case("prompt_1b_512", "prompt", 1, 64, 0, tokens=512),
        # prompts of 500 to 4,001 tokens of a serving batch, some after a chat, 8B shape
        case("prompt_8b_packed", "prompt", 7, 128, 900, tokens=4001),
        # a chunk of a long prompt, 8B shape: the largest call
        case("prompt_8b_chunk", "prompt", 1, 128, 30720, tokens=2048, page=64),
        # one more token for each sequence of a full batch: a few of them need a page
        case("advance_8b_b32", "advance", 32, 128, 2049, tokens=1),
        # a step of eight beam searches of four beams each, all layers of the 1B shape: beams that go on twice share a page
        case("advance_beams", "advance", 32, 64, 700, tokens=1, page=64, layers=16, beams=4),
        # the tiny fp32 model's pool
        case("compact_tiny_f32", "compact", 3, 64, 200, dtype="f32", H=4, Hk=2, page=16, layers=2),
        # a serving pool of four layers after many sequences have come and gone
        case("compact_8b", "compact", 32, 128, 2600, layers=4),
    ]


def draw(rng):
    def spread(lo, hi):  # over the logarithm, odd sizes among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(("append", "attn", "attn", "prompt", "prompt", "prompt", "advance", "compact"))
    H, Hk = rng.choice(((32, 8), (32, 8), (4, 2), (8, 8), (9, 3), (32, 4), (16, 1)))
    rows = spread(1, 64)
    c = {"kind": kind, "dtype": "f32" if rng.random() < 0.2 else "bf16", "rows": rows, "H": H, "Hk": Hk,
         "hd": rng.choice((64, 128)), "page": rng.choice((16, 32, 32, 64, 128, 256)), "kv": 0, "tokens": 0, "layers": 1, "beams": 0}
    if kind == "append":
        c.update(tokens=spread(1, 16000 // rows), kv=spread(1, 2000))
    elif kind == "attn":
        c["kv"] = spread(1, min(33000, 130000 // rows))
    elif kind == "prompt":
        scores = 1_000_000_000 // (rows * H) // (4 if c["dtype"] == "f32" else 1)   # of a (row, q-head), padded
        tokens = spread(1, min(4000, math.isqrt(scores)))
        c.update(tokens=tokens, kv=rng.choice((0, spread(1, max(1, min(33000, 130000 // rows, scores // tokens - tokens))))))
    else:
        c.update(layers=spread(1, 16), kv=spread(20, min(5000, 20000 // rows)))
        if kind == "advance":
            c.update(tokens=spread(1, 64), beams=rng.choice((0, 2, 4)))
            if c["beams"]:
                c["rows"] = max(1, rows // c["beams"]) * c["beams"]
        slots = 2 * rows * (c["kv"] + c["tokens"] + 2 * c["page"])  # what the pool may have
        c["layers"] = max(1, min(c["layers"], 600_000_000 // (slots * Hk * c["hd"] * 4)))
    return c


# ---------------------------------------------------------------- lengths
def _spread(longest, rows, least):
    """`rows` lengths from `longest` down to about `least` of it, over the logarithm."""
    return [max(1, round(longest * least ** (i / max(1, rows - 1)))) if longest else 0 for i in range(rows)]


def _sizes(case):
    """(slots held, new tokens) of each row, the rows in no particular order of a batch."""
    R, kv, T = case["rows"], case["kv"], case["tokens"]
    if case["kind"] in ("append", "prompt"):
        return [(round(kv * ((i * 5) % R) / max(1, R - 1)) if R > 1 else kv, t) for i, t in enumerate(_spread(T, R, 0.125))]
    if case["kind"] == "advance" and case["beams"]:   # the beams of a search are equally long
        return [(n, T) for n in _spread(kv, R // case["beams"], 0.7) for _ in range(case["beams"])]
    return [(n, T) for n in _spread(kv, R, 0.8)]


def _pages(n, P):
    return (n + P - 1) // P


def _capacity(case):
    """Table entries of a row, pages of the pool."""
    P, sizes = case["page"], _sizes(case)
    row_pages = _pages(max(n + t for n, t in sizes), P) + 1
    held = sum(_pages(n + t, P) for n, t in sizes)
    return row_pages, held + held // 2 + case["rows"] + 1


# ---------------------------------------------------------------- the pool
def _storage(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _unit(case):
    return 4 if case["dtype"] == "f32" else 8   # values of 16 bytes


def _to_page(k, v, case):
    """K and V [..., page, hd] in the order of the pool, [..., 2, page * hd]."""
    lead, P, hd, E = k.shape[:-2], case["page"], case["hd"], _unit(case)
    n = len(lead)
    k = k.reshape(*lead, P // 16, 2, 2, 4, hd // E, E).permute(*range(n), n, n + 4, n + 2, n + 1, n + 3, n + 5).reshape(*lead, P * hd)
    v = v.reshape(*lead, P // E, E, hd).transpose(n + 1, n + 2).reshape(*lead, P * hd)
    return torch.stack([k, v], n)


def _from_page(x, case):
    """The inverse of _to_page."""
    lead, P, hd, E = x.shape[:-2], case["page"], case["hd"], _unit(case)
    n = len(lead)
    k, v = x[..., 0, :], x[..., 1, :]
    k = k.reshape(*lead, P // 16, hd // E, 2, 2, 4, E).permute(*range(n), n, n + 3, n + 2, n + 4, n + 1, n + 5).reshape(*lead, P, hd)
    v = v.reshape(*lead, P // E, hd, E).transpose(n + 1, n + 2).reshape(*lead, P, hd)
    return k, v


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


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _metadata(case, g, lens, held):
    """One int32 buffer of slots held, tables and reference counts, and its views; tables of pages in no order."""
    R, P = case["rows"], case["page"]
    row_pages, n_pages = _capacity(case)
    meta = torch.full((R + R * row_pages + n_pages,), -1, dtype=torch.int32, device=DEV)
    kv_len, table, refs = meta[:R], meta[R:R + R * row_pages].view(R, row_pages), meta[R + R * row_pages:]
    kv_len.copy_(lens)
    ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    n = (held + P - 1) // P
    at = n.cumsum(0) - n
    e = torch.arange(row_pages, device=DEV)
    table.copy_(torch.where(e < n[:, None], ids[(at[:, None] + e).clamp(max=n_pages - 1)], table))
    if case["beams"]:   # the first six of seven pages are the prompt's, which the beams share
        first = torch.arange(R, device=DEV) // case["beams"] * case["beams"]
        table.copy_(torch.where(e < (n * 6 // 7)[:, None], table[first], table))
    refs.copy_(_count(table, n, n_pages))
    return meta, kv_len, table, refs


def prepare(case, seed):
    g = _rng(seed)
    R, H, Hk, hd, P = case["rows"], case["H"], case["Hk"], case["hd"], case["page"]
    row_pages, n_pages = _capacity(case)
    sizes = torch.tensor(_sizes(case), device=DEV)
    if not case["beams"]:
        sizes = sizes[torch.randperm(R, generator=g, device=DEV)]
    start, count = sizes[:, 0], sizes[:, 1]
    held = start if case["kind"] in ("attn", "advance", "compact") else start + count

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    s = {"case": case, "err": torch.zeros(R, dtype=torch.int32, device=DEV),
         "ws": torch.zeros(_workspace_bytes(case), dtype=torch.uint8, device=DEV)}
    lens = start if case["kind"] in ("append", "advance", "compact") else held
    s["meta"], s["kv_len"], s["table"], s["refs"] = _metadata(case, g, lens, held)
    # keys with channels of unequal size and mean, values of unequal size
    t = _storage(case)
    size, mean = torch.exp(0.5 * randn(Hk, 1, hd)), randn(Hk, 1, hd)
    s["pool"] = torch.empty(case["layers"], n_pages, Hk, 2, P * hd, dtype=t, device=DEV)
    for layer in s["pool"]:
        K, V = randn(n_pages, Hk, P, hd).add_(mean).mul_(0.6 * size), randn(n_pages, Hk, P, hd)
        layer.copy_(_to_page(K.to(t), V.to(t), case))
        del K, V
    offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0)).to(torch.int32)
    N = sum(n for _, n in _sizes(case))
    if case["kind"] == "append":
        s["offsets"] = offsets
        s["qkv"] = randn(N, (H + 2 * Hk) * hd)
        row = torch.bucketize(torch.arange(N, device=DEV), offsets[1:].long(), right=True)
        pos = start[row] + torch.arange(N, device=DEV) - offsets[row]
        angle = pos[:, None].double() * 500000.0 ** (-2.0 * torch.arange(hd // 2, device=DEV).double() / hd)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q"] = torch.zeros(N, H * hd * (1 if case["dtype"] == "f32" else 2), dtype=t, device=DEV)
    elif case["kind"] in ("attn", "prompt"):
        s["q"] = _act(1.5 * randn(N if case["kind"] == "prompt" else R, H * hd), case)
        s["out"] = torch.zeros_like(s["q"])
        s["on"] = torch.ones(R, dtype=torch.int32, device=DEV)
        s["offsets"], s["kv_max"] = offsets, max(n + t for n, t in _sizes(case))
    else:
        # a pass starts from the tables of the step, which a scheduler hands over: they are put back at its start
        s["meta0"] = s["meta"].clone()
        s["start"] = torch.zeros(R, dtype=torch.int32, device=DEV)
        s["count"] = count.to(torch.int32)
        s["parent"] = None
        if case["beams"]:   # each beam goes on with one of its search's beams
            b = case["beams"]
            best = torch.randint(0, b, (R // b, b), generator=g, device=DEV)
            s["parent"] = (best + b * torch.arange(R // b, device=DEV)[:, None]).view(R).to(torch.int32)
        s["map"] = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        s["used"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _workspace_bytes(case):
    """What a caller keeps for the kernels' intermediate records: at least ham_op_paged_workspace_bytes."""
    row_pages, n_pages = _capacity(case)
    R, pairs, group = case["rows"], case["rows"] * case["Hk"], case["H"] // case["Hk"]
    return max((2048 + 5 * pairs) * group, 1 << 17) * (case["hd"] + 2) * 4 + (R * row_pages + 4 * n_pages + 16 * R) * 4 + (1 << 16)


# ---------------------------------------------------------------- one pass, plain
def _rope(x, cos, sin):
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _rows_of(s, N):
    """Row and place within the row of each packed token."""
    i = torch.arange(N, device=DEV)
    row = torch.bucketize(i, s["offsets"][1:].long(), right=True).clamp(max=s["case"]["rows"] - 1)
    return row, i - s["offsets"][row]


def _plain_append(s):
    case = s["case"]
    H, Hk, hd, P, E = case["H"], case["Hk"], case["hd"], case["page"], _unit(case)
    N = s["qkv"].shape[0]
    x = s["qkv"].view(N, H + 2 * Hk, hd)
    cos, sin = s["cos"][:, None], s["sin"][:, None]
    s["q"].copy_(_act(_rope(x[:, :H], cos, sin).view(N, H * hd), case))
    row, i = _rows_of(s, N)
    slot = s["kv_len"][row] + i
    page = s["table"][row, slot // P].long()
    at = (slot % P).long()[:, None]
    d = torch.arange(hd, device=DEV)
    k_at = ((at // 16 * (hd // E) + d // E) * 16 + at // 4 % 2 * 8 + at // 8 % 2 * 4 + at % 4) * E + d % E
    v_at = (at // E * hd + d) * E + at % E
    first = (page[:, None] * Hk + torch.arange(Hk, device=DEV))[..., None] * (2 * P * hd)
    pool = s["pool"].view(-1)
    pool[first + k_at[:, None]] = _rope(x[:, H:H + Hk], cos, sin).to(pool.dtype)
    pool[first + P * hd + v_at[:, None]] = x[:, H + Hk:].to(pool.dtype)
    return {"q": s["q"], "pool": s["pool"], "err": s["err"]}


def _gathered(s):
    """K and V of every table entry of each row in fp32, [R][Hk][row_pages * P][hd]."""
    case = s["case"]
    R, Hk, hd, P = case["rows"], case["Hk"], case["hd"], case["page"]
    k, v = _from_page(s["pool"][0][s["table"].clamp(min=0).long()], case)   # [R][row_pages][Hk][P][hd]
    return (x.float().transpose(1, 2).reshape(R, Hk, -1, hd) for x in (k, v))


def _attend(q, K, V, seen):
    """q [R][Hk][n][hd] over K, V [R][Hk][S][hd]; seen broadcasts to [R][Hk][n][S]."""
    sc = (q @ K.transpose(2, 3)).masked_fill_(~seen, -math.inf)
    sc = sc.sub_(sc.amax(-1, keepdim=True)).exp_()
    return (sc @ V) / sc.sum(-1, keepdim=True)


def _plain_attention(s):
    case = s["case"]
    R, H, Hk, hd = case["rows"], case["H"], case["Hk"], case["hd"]
    K, V = _gathered(s)
    q = _from_act(s["q"], case).view(R, Hk, H // Hk, hd) / math.sqrt(hd)
    seen = torch.arange(K.shape[2], device=DEV) < s["kv_len"][:, None, None, None]
    s["out"].copy_(_act(_attend(q, K, V, seen).view(R, H * hd), case))
    return {"out": s["out"], "err": s["err"]}


def _plain_prompt(s):
    case = s["case"]
    R, H, Hk, hd, T = case["rows"], case["H"], case["Hk"], case["hd"], case["tokens"]
    N, grp = s["q"].shape[0], H // Hk
    K, V = _gathered(s)
    count = s["offsets"][1:] - s["offsets"][:-1]
    t = torch.arange(T, device=DEV)
    tok = (s["offsets"][:-1, None] + t).clamp(max=N - 1).long()
    q = _from_act(s["q"], case)[tok].view(R, T, Hk, grp, hd).permute(0, 2, 3, 1, 4).reshape(R, Hk, grp * T, hd) / math.sqrt(hd)
    last = (s["kv_len"] - count)[:, None] + t                   # the last slot that a token sees
    seen = torch.arange(K.shape[2], device=DEV) <= last[..., None]
    o = _attend(q, K, V, seen[:, None].repeat(1, 1, grp, 1))
    row, i = _rows_of(s, N)
    o = o.view(R, Hk, grp, T, hd)[row, :, :, i].reshape(N, H * hd)
    s["out"].copy_(_act(o, case))
    return {"out": s["out"], "err": s["err"]}


def _count(table, n, n_pages):
    """How many of the first n[r] entries of each row name a page."""
    e = torch.arange(table.shape[1], device=DEV)
    at = torch.where(e < n[:, None], table, torch.full_like(table, n_pages)).long().view(-1)
    return torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV).scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:n_pages]


def _plain_advance(s):
    case, P, R = s["case"], s["case"]["page"], s["case"]["rows"]
    s["meta"].copy_(s["meta0"])
    n_pages = s["refs"].shape[0]
    r, e = torch.arange(R, device=DEV), torch.arange(s["table"].shape[1], device=DEV)
    had = _pages(s["kv_len"].long(), P)
    source = r if s["parent"] is None else s["parent"].long()
    length, table, c = s["kv_len"].long()[source], s["table"][source], s["count"].long()
    held = _pages(length, P)
    refs = _count(table, held, n_pages)
    # a page that is written to and that another row holds: the lowest row keeps it where all that hold it write to it
    last = (held - 1).clamp(min=0)
    page = table.gather(1, last[:, None])[:, 0].long().clamp(min=0)
    shared = (c > 0) & (length % P > 0) & (refs[page] > 1)
    at = torch.where(shared, page, torch.full_like(page, n_pages))
    writers = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV).scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    lowest = torch.full((n_pages + 1,), R, dtype=torch.int64, device=DEV).scatter_reduce_(0, at, r, "amin")
    copied = shared & ~((writers[at] == refs[page]) & (lowest[at] == r))
    need = _pages(length + c, P) - held + copied
    end = need.cumsum(0)
    enough = end[-1] <= (refs == 0).sum()
    free = torch.sort((refs > 0).to(torch.int32), stable=True).indices
    copied, c = copied & enough, torch.where(enough, c, torch.zeros_like(c))
    first = torch.where(enough, end - need, torch.zeros_like(end))
    mine = free[(first[:, None] + (e - held[:, None] + copied[:, None])).clamp(0, n_pages - 1)]
    now = _pages(length + c, P)
    new = (e >= held[:, None]) & (e < now[:, None])
    new |= copied[:, None] & (e == last[:, None])
    table = torch.where(new, mine.to(torch.int32), table)
    table = torch.where(e < now[:, None], table, torch.where(e < had[:, None], torch.full_like(table, -1), s["table"]))
    to = torch.where(copied, mine.gather(1, last[:, None])[:, 0], page)
    s["pool"][:, to] = s["pool"][:, page]
    s["table"].copy_(table)
    s["kv_len"].copy_(length + c)
    s["start"].copy_(length)
    s["refs"].copy_(_count(table, now, n_pages))
    s["err"].copy_(torch.where((s["count"] > 0) & ~enough, s["err"] | 64, s["err"]))
    return {"kv_len": s["kv_len"], "start": s["start"], "table": s["table"], "refs": s["refs"], "pool": s["pool"], "err": s["err"]}


def _plain_compact(s):
    P = s["case"]["page"]
    s["meta"].copy_(s["meta0"])
    p = torch.arange(s["refs"].shape[0], device=DEV)
    live = s["refs"] > 0
    used = live.sum()
    holes = torch.sort((live | (p >= used)).to(torch.int32), stable=True).indices    # free pages below `used` first
    moves = live & (p >= used)
    to = torch.where(moves, holes[(moves.long().cumsum(0) - 1).clamp(min=0)], p)
    source = torch.full((p.numel() + 1,), -1, dtype=torch.int64, device=DEV)
    source.scatter_(0, torch.where(moves, to, torch.full_like(to, p.numel())), p)
    source = torch.where(source[:-1] >= 0, source[:-1], p)
    s["pool"].copy_(s["pool"].index_select(1, source))
    s["map"].copy_(torch.where(live, to, torch.full_like(to, -1)))
    s["refs"].copy_(torch.where(p < used, s["refs"][source], torch.zeros_like(s["refs"])))
    e = torch.arange(s["table"].shape[1], device=DEV)
    holds = e < _pages(s["kv_len"].long(), P)[:, None]
    s["table"].copy_(torch.where(holds, s["map"][s["table"].clamp(min=0).long()], s["table"]))
    s["used"].copy_(used)
    return {"table": s["table"], "refs": s["refs"], "map": s["map"], "used": s["used"], "pool": s["pool"], "err": s["err"]}


def _kernels(s):
    from paper_2505_20438_amd import ham
    case = s["case"]
    row_pages, n_pages = s["table"].shape[1], s["refs"].shape[0]
    shape = ham.paged_shape(ham.HAM_F32 if case["dtype"] == "f32" else ham.HAM_BF16, case["rows"], case["H"], case["Hk"],
                            case["hd"], case["page"], n_pages, row_pages)
    stream = torch.cuda.current_stream().cuda_stream
    kind = case["kind"]
    if kind == "append":
        ham.ham_op_paged_append(shape, s["qkv"], s["cos"], s["sin"], s["offsets"], s["kv_len"], s["table"], s["pool"], s["q"], s["err"],
                                stream)
        return {"q": s["q"], "pool": s["pool"], "err": s["err"]}
    if kind == "attn":
        ham.ham_op_paged_attention(shape, s["q"], s["pool"], s["table"], s["kv_len"], s["on"], s["kv_max"], s["out"], s["err"], s["ws"],
                                   stream)
        return {"out": s["out"], "err": s["err"]}
    if kind == "prompt":
        ham.ham_op_paged_prompt(shape, s["q"], s["offsets"], s["pool"], s["table"], s["kv_len"], s["kv_max"], s["out"], s["err"], s["ws"],
                                stream)
        return {"out": s["out"], "err": s["err"]}
    s["meta"].copy_(s["meta0"])
    if kind == "advance":
        ham.ham_op_paged_advance(shape, case["layers"], s["parent"], s["count"], s["kv_len"], s["start"], s["table"], s["refs"], s["pool"],
                                 s["err"], s["ws"], stream)
        return {"kv_len": s["kv_len"], "start": s["start"], "table": s["table"], "refs": s["refs"], "pool": s["pool"], "err": s["err"]}
    ham.ham_op_paged_compact(shape, case["layers"], s["kv_len"], s["table"], s["refs"], s["pool"], s["map"], s["used"], s["err"], s["ws"],
                             stream)
    return {"table": s["table"], "refs": s["refs"], "map": s["map"], "used": s["used"], "pool": s["pool"], "err": s["err"]}


def run(state):
    if own:
        return _kernels(state)
    return {"append": _plain_append, "attn": _plain_attention, "prompt": _plain_prompt, "advance": _plain_advance,
            "compact": _plain_compact}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- work
def work(case):
    R, H, Hk, hd, P = case["rows"], case["H"], case["Hk"], case["hd"], case["page"]
    es = 4 if case["dtype"] == "f32" else 2
    sizes = _sizes(case)
    N, act = sum(t for _, t in sizes), 4 * H * hd
    if case["kind"] == "append":
        return {"bytes": N * (4 * (H + 2 * Hk) * hd + 4 * hd + act + 2 * Hk * hd * es), "flops": N * 3.0 * (H + Hk) * hd}
    if case["kind"] == "attn":
        kv = sum(n for n, _ in sizes)
        return {"bytes": kv * Hk * 2 * hd * es + 2 * R * act, "flops": 4.0 * kv * H * hd}
    if case["kind"] == "prompt":
        kv = sum(n + t for n, t in sizes)
        return {"bytes": kv * Hk * 2 * hd * es + 2 * N * act, "flops": 4.0 * H * hd * sum(t * n + t * (t + 1) / 2 for n, t in sizes)}
    row_pages, n_pages = _capacity(case)
    page = case["layers"] * Hk * 2 * P * hd * es
    held = sum(_pages(n, P) for n, _ in sizes)
    if case["kind"] == "advance":
        b = case["beams"]
        copied = 0
        if b:   # beams that go on twice: all but one of them copy, where the last page is not full
            copied = b * (1 - 1 / b) ** b * sum(1 for n, _ in sizes if n % P) / b
        return {"bytes": 8 * held + 4 * n_pages + 2 * copied * page, "flops": 2.0 * held}
    moved = held * (n_pages - held) / n_pages   # of pages in no order
    return {"bytes": 8 * held + 8 * n_pages + 2 * moved * page, "flops": 1.0 * n_pages}


# ---------------------------------------------------------------- float64
def _stored64(x, case):
    return x.float().to(_storage(case)).double()


def _pair64(x, case):
    if case["dtype"] == "f32":
        return x
    hi = _stored64(x, case)
    return torch.cat([hi, _stored64(x - hi, case)], -1)


def _row64(s, r, n):
    """K and V [Hk][n][hd] of the first n slots of row r in float64, by the formulas of the layout."""
    case = s["case"]
    hd, P, E = case["hd"], case["page"], _unit(case)
    i, d = torch.arange(n, device=DEV), torch.arange(hd, device=DEV)[None]
    pages, at = s["table"][r].long()[i // P], (i % P)[:, None]
    place = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device=DEV)[at % 16]
    k = ((at // 16 * (hd // E) + d // E) * 16 + place) * E + d % E
    v = (at // E * hd + d) * E + at % E
    x = s["pool"][0][pages]                                      # [n][Hk][2][P * hd]
    x = torch.stack([x[:, :, 0].gather(2, k[:, None].expand(n, case["Hk"], hd)), x[:, :, 1].gather(2, v[:, None].expand(n, case["Hk"], hd))])
    return x.double().transpose(1, 2)


def exact(case, seed):
    if case["kind"] in ("advance", "compact"):
        return None  # whole numbers and copies
    s = prepare(case, seed)
    R, H, Hk, hd, P, E = case["rows"], case["H"], case["Hk"], case["hd"], case["page"], _unit(case)
    grp = H // Hk
    lens, off = s["kv_len"].tolist(), s["offsets"].tolist()
    if case["kind"] == "append":
        x = s["qkv"].double().view(-1, H + 2 * Hk, hd)
        c, sn = s["cos"].double()[:, None], s["sin"].double()[:, None]
        a, b = x[..., :hd // 2], x[..., hd // 2:]

        def f32(y):  # an fp32 operation of the definition rounds
            return y.float().double()
        rot = torch.cat([f32(f32(a * c) - f32(b * sn)), f32(f32(b * c) + f32(a * sn))], -1)
        pool = s["pool"].double()
        place = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device=DEV)
        for r in range(R):
            n = off[r + 1] - off[r]
            slot = lens[r] + torch.arange(n, device=DEV)
            pages, at = s["table"][r].long()[slot // P], slot % P
            kv = _stored64(rot[off[r]:off[r + 1], H:H + Hk], case), _stored64(x[off[r]:off[r + 1], H + Hk:], case)
            for d in range(hd):
                pool[0][pages, :, 0, ((at // 16 * (hd // E) + d // E) * 16 + place[at % 16]) * E + d % E] = kv[0][..., d]
                pool[0][pages, :, 1, (at // E * hd + d) * E + at % E] = kv[1][..., d]
        return {"q": _pair64(rot[:, :H].reshape(-1, H * hd), case), "pool": pool, "err": None}
    q = _from_act(s["q"], case).double().view(-1, H, hd)
    o = torch.zeros_like(q)
    for r in range(R):
        n = lens[r]
        i = slice(r, r + 1) if case["kind"] == "attn" else slice(off[r], off[r + 1])
        K, V = _row64(s, r, n)
        last = torch.arange(n - q[i].shape[0], n, device=DEV)
        hidden = torch.arange(n, device=DEV) > last[:, None]
        for h in range(H):
            sc = (q[i, h] @ K[h // grp].T / math.sqrt(hd)).masked_fill_(hidden, -math.inf)
            o[i, h] = torch.softmax(sc, -1) @ V[h // grp]
    return {"out": _pair64(o.view(-1, H * hd), case), "err": None}
