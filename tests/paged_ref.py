"""The paged KV cache and the operators over it on the CPU, from their definition in include/ham_ops.h: attention in float64,
pool contents rounded where the definition rounds, tables and references as plain lists, row by row.

Tolerances.  Pool contents, rotated q, tables, references and maps are held to the definition bit for bit.  Attention: FILLED_TOL
of attention_bounds.py, which a lost or doubled slot exceeds, and the bound of kv8_planes.py, KAPPA |S| + OUT |out|: its derivation
holds here as it stands (queries of standard deviation SIGMA_Q, keys and values of 1, weights of 24 significant bits, without the
scales of an 8-bit cache).  In bf16 a lost plane of the weights exceeds it on the inputs with pairs of paged_planes.py; on independent
values, as rows_of_pages of test_gpu_paged.py makes them, the output's rounding covers most of it (0.8 to 1.1 of the bound).
"""
import torch

from tests.kv8_ref import rope64, storage, stored  # noqa: F401


def places(P, hd, E):
    """Where K and V of (slot, channel) are within a page's K, or V, of a kv head."""
    s, d = torch.arange(P)[:, None], torch.arange(hd)[None]
    k = ((s // 16 * (hd // E) + d // E) * 16 + s // 4 % 2 * 8 + s // 8 % 2 * 4 + s % 4) * E + d % E
    return k, (s // E * hd + d) * E + s % E


class Pool:
    """Layers' pools [layers][n_pages][n_kv_heads][2][P * hd] on the CPU, tables and references."""

    def __init__(self, shape, layers=1, fill=None):
        self.s, self.layers = shape, layers
        t = storage(shape.dtype)
        self.E = 8 if t == torch.bfloat16 else 4
        dims = (layers, shape.n_pages, shape.n_kv_heads, 2, shape.page_slots * shape.head_dim)
        n = 1
        for x in dims:
            n *= x
        bytes_ = torch.full((n * t.itemsize,), 0xAB if fill is None else fill, dtype=torch.uint8)
        self.data = bytes_.view(t).view(dims)
        self.ki, self.vi = places(shape.page_slots, shape.head_dim, self.E)
        self.table = [[-1] * shape.row_pages for _ in range(shape.rows)]
        self.refs = [0] * shape.n_pages
        self.len = [0] * shape.rows

    def pages(self, n):
        return -(-n // self.s.page_slots)

    # ---- contents
    def append(self, r, start, k, v, layer=0):
        """k, v [n][kv heads][hd] of stored values (float64)."""
        P = self.s.page_slots
        for i in range(k.shape[0]):
            page, at = self.table[r][(start + i) // P], (start + i) % P
            self.data[layer, page, :, 0, self.ki[at]] = k[i].to(self.data.dtype)
            self.data[layer, page, :, 1, self.vi[at]] = v[i].to(self.data.dtype)

    def keys_values(self, r, n, layer=0):
        """K, V [kv heads][n][hd] in float64."""
        m = self.pages(n)
        x = self.data[layer, self.table[r][:m]].double()                   # [m][Hk][2][P * hd]
        out = [x[:, :, j][:, :, at].transpose(0, 1).reshape(self.s.n_kv_heads, -1, self.s.head_dim)[:, :n] for j, at in ((0, self.ki), (1, self.vi))]
        return out if m else [torch.zeros(self.s.n_kv_heads, 0, self.s.head_dim, dtype=torch.float64)] * 2

    # ---- attention
    def attention(self, q, lens):
        """One query row of each sequence, q float64 [rows][H][hd]."""
        out, spread = torch.zeros_like(q), torch.zeros_like(q)
        for r, n in enumerate(lens):
            if n > 0:
                out[r:r + 1], spread[r:r + 1] = self._attend(r, q[r:r + 1], n)
        return out, spread

    def prompt(self, q, offsets, lens):
        out, spread = torch.zeros_like(q), torch.zeros_like(q)
        for r, n in enumerate(lens):
            i = slice(offsets[r], offsets[r + 1])
            if offsets[r + 1] > offsets[r]:
                out[i], spread[i] = self._attend(r, q[i], n)
        return out, spread

    def _attend(self, r, q, n):
        """The last q.shape[0] of n slots see those up to their own: outputs, and S with S_d^2 = sum (p v_d)^2."""
        c, H, hd = q.shape
        Hk = self.s.n_kv_heads
        k, v = self.keys_values(r, n)
        hidden = torch.arange(n) > (n - c + torch.arange(c))[:, None]
        out, spread = torch.zeros_like(q), torch.zeros_like(q)
        for h in range(H):
            p = torch.softmax((q[:, h] @ k[h * Hk // H].T / hd ** 0.5).masked_fill(hidden, -float("inf")), -1)
            out[:, h], spread[:, h] = p @ v[h * Hk // H], (p.square() @ v[h * Hk // H].square()).sqrt()
        return out, spread

    # ---- bookkeeping
    def advance(self, parent, count):
        """-> (start, err), and the change of contents, tables, references and lengths."""
        R, P, cap = self.s.rows, self.s.page_slots, self.s.row_pages * self.s.page_slots
        err = [0] * R
        old, lens = [list(t) for t in self.table], list(self.len)
        if parent is not None:
            for r in range(R):
                p = parent[r]
                if p < -1 or p >= R:
                    err[r], p = err[r] | 8, r
                if p == r:
                    continue
                had, now = self.pages(lens[r]), 0 if p < 0 else self.pages(lens[p])
                for e in range(had):
                    self.refs[old[r][e]] -= 1
                for e in range(now):
                    self.refs[old[p][e]] += 1
                self.table[r][:now] = old[p][:now] if p >= 0 else []
                self.table[r][now:had] = [-1] * max(0, had - now)
                self.len[r] = lens[p] if p >= 0 else 0
        change = []
        for r in range(R):
            fits = 0 <= self.len[r] + count[r] <= cap
            err[r] |= 0 if fits else 8
            change.append(count[r] if fits else 0)
        for r in range(R):
            if change[r] < 0:
                for e in range(self.pages(self.len[r] + change[r]), self.pages(self.len[r])):
                    self.refs[self.table[r][e]] -= 1
                    self.table[r][e] = -1
        last = [self.table[r][self.len[r] // P] if change[r] > 0 and self.len[r] % P else -1 for r in range(R)]
        writers = {p: [r for r in range(R) if last[r] == p] for p in set(last) - {-1}}
        copied = [last[r] >= 0 and self.refs[last[r]] > 1 and not (len(writers[last[r]]) == self.refs[last[r]] and writers[last[r]][0] == r)
                  for r in range(R)]
        free = [p for p in range(self.s.n_pages) if self.refs[p] <= 0]
        need = [self.pages(self.len[r] + change[r]) - self.pages(self.len[r]) + copied[r] if change[r] > 0 else 0 for r in range(R)]
        start = [0] * R
        enough = sum(need) <= len(free)
        for r in range(R):
            if change[r] > 0 and not enough:
                err[r] |= 64
                change[r] = 0
            start[r] = self.len[r] + min(change[r], 0)
            if change[r] > 0:
                held = self.pages(self.len[r])
                if copied[r]:
                    p = free.pop(0)
                    self.refs[last[r]] -= 1
                    self.refs[p] = 1
                    self.table[r][held - 1] = p
                    self.data[:, p] = self.data[:, last[r]]
                for e in range(held, self.pages(self.len[r] + change[r])):
                    self.table[r][e] = free.pop(0)
                    self.refs[self.table[r][e]] = 1
            self.len[r] += change[r]
        return start, err

    def compact(self):
        """-> (map, pages in use)."""
        live = [p for p in range(self.s.n_pages) if self.refs[p] > 0]
        used = len(live)
        holes = [p for p in range(used) if self.refs[p] <= 0]
        to = {p: p for p in live}
        for p, hole in zip((p for p in live if p >= used), holes):
            to[p] = hole
            self.data[:, hole] = self.data[:, p]
            self.refs[hole], self.refs[p] = self.refs[p], 0
        for r in range(self.s.rows):
            m = self.pages(self.len[r])
            self.table[r][:m] = [to[p] for p in self.table[r][:m]]
        return [to.get(p, -1) for p in range(self.s.n_pages)], used

    def sound(self):
        """Whether the references are those of the tables and no two rows share a page by mistake of the test."""
        n = [0] * self.s.n_pages
        for r in range(self.s.rows):
            for e in range(self.pages(self.len[r])):
                n[self.table[r][e]] += 1
        return n == [max(0, x) for x in self.refs]
