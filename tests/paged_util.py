"""A K/V cache in pages in plain Python: every call of the library's one entry and one page at a time, values in 64 bits."""
import torch

EINVAL, ECAPACITY = -1, -3


def canonical(pool, Dh):
    """[layers][pages][heads][blocks][32 * Dh] in the library's K and V order -> two readings [layers][pages][heads][positions][Dh]."""
    L, N, H, PB, _ = pool.shape
    G = Dh // 32
    p, d = torch.arange(32)[:, None], torch.arange(Dh)[None]
    k = ((p // 4 % 2 * 4 + d % 32 // 8) * 16 * G + 4 * (p // 8) + p % 4 + 16 * (d // 32)) * 8 + d % 8
    v = (d // 16 * 64 + d % 16 + 16 * (p // 8)) * 8 + p % 8
    return [pool[..., i.reshape(-1).to(pool.device)].view(L, N, H, PB * 32, Dh) for i in (k, v)]


class Plain:
    """The book as lists; K and V as the library's pools, read by canonical()."""

    def __init__(self, cache):
        d = cache._desc
        self.P, self.S, self.MP, self.N = d.page_size, d.max_seqs, d.max_pages, d.n_pages
        self.table, self.len, self.ref = cache.table.tolist(), cache.len.tolist(), cache.ref.tolist()
        self.k, self.v = cache.k.clone(), cache.v.clone()

    def same(self, cache):
        assert cache.table.tolist() == self.table and cache.len.tolist() == self.len and cache.ref.tolist() == self.ref
        bits = torch.int16 if cache.k.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(cache.k.view(bits), self.k.view(bits)) and torch.equal(cache.v.view(bits), self.v.view(bits))
        for p in range(self.N):
            assert self.ref[p] == sum(row.count(p) for row in self.table)

    def _slots(self, s, rows):
        return range(self.len[s] // self.P, -(-(self.len[s] + rows) // self.P))

    def _free_pages(self):
        return [p for p in range(self.N) if self.ref[p] == 0]

    def grow(self, seqs, rows):
        status, asked, free = [], 0, self._free_pages()
        for i, (s, r) in enumerate(zip(seqs, rows)):
            if not 0 <= s < self.S or r < 0 or s in seqs[:i]:
                status.append(EINVAL)
                continue
            slots = self._slots(s, r)
            if slots.stop > self.MP:
                status.append(ECAPACITY)
                continue
            want = [k for k in slots if self.table[s][k] < 0]
            asked += len(want)
            if want and asked > len(free):
                status.append(ECAPACITY)
                continue
            for k, p in zip(want, free[asked - len(want):]):
                self.table[s][k], self.ref[p] = p, 1
            status.append(0)
        return status

    def advance(self, seqs, rows):
        status = []
        for i, (s, r) in enumerate(zip(seqs, rows)):
            if not 0 <= s < self.S or r < 0 or s in seqs[:i]:
                status.append(EINVAL)
                continue
            slots = self._slots(s, r)
            ok = slots.stop <= self.MP and all(self.table[s][k] >= 0 for k in slots)
            status.append(0 if ok else ECAPACITY)
            self.len[s] += r if ok else 0
        return status

    def fork(self, src, dst):
        status, asked, free = [], 0, self._free_pages()
        empty = [n == 0 and row[0] < 0 for n, row in zip(self.len, self.table)]
        for i, (s, d) in enumerate(zip(src, dst)):
            if not (0 <= s < self.S and 0 <= d < self.S) or d in dst[:i] or s in dst or not empty[d]:
                status.append(EINVAL)
                continue
            last, part = divmod(self.len[s], self.P)
            own = part > 0 and self.table[s][last] >= 0
            asked += own
            if own and asked > len(free):
                status.append(ECAPACITY)
                continue
            for k in range(last):
                p = self.table[d][k] = self.table[s][k]
                if p >= 0:
                    self.ref[p] += 1
            if own:
                p, old, blocks = free[asked - 1], self.table[s][last], -(-part // 32)
                self.table[d][last], self.ref[p] = p, 1
                for pool in (self.k, self.v):
                    pool[:, p, :, :blocks] = pool[:, old, :, :blocks]
            self.len[d] = self.len[s]
            status.append(0)
        return status

    def _leave(self, s, k):
        p, self.table[s][k] = self.table[s][k], -1
        if p >= 0:
            self.ref[p] -= 1

    def trim(self, seqs, window, sinks):
        for s in seqs:
            if 0 <= s < self.S:
                for k in range(self.MP):
                    if k * self.P >= sinks and (k + 1) * self.P - 1 <= self.len[s] - window:
                        self._leave(s, k)
        return [0 if 0 <= s < self.S else EINVAL for s in seqs]

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < self.S:
                for k in range(self.MP):
                    self._leave(s, k)
                self.len[s] = 0
        return [0 if 0 <= s < self.S else EINVAL for s in seqs]

    def compact(self):
        used = sum(r > 0 for r in self.ref)
        src, dst = [p for p in range(used, self.N) if self.ref[p]], [p for p in range(used) if not self.ref[p]]
        to = dict(zip(src, dst))
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        for s, d in to.items():
            self.ref[d], self.ref[s] = self.ref[s], 0
            for pool in (self.k, self.v):
                pool[:, d] = pool[:, s]
        return used

    def write(self, Dh, layer, seqs, rows, k, v):
        """rows[i] rows of sequence seqs[i], one sequence after the other."""
        kc, vc = canonical(self.k, Dh)[0], canonical(self.v, Dh)[1]
        kp, vp, x = kc.clone(), vc.clone(), 0
        for s, r in zip(seqs, rows):
            for j in range(r):
                slot, p = divmod(self.len[s] + j, self.P) if 0 <= s < self.S else (self.MP, 0)
                if slot < self.MP and self.table[s][slot] >= 0:
                    kp[layer, self.table[s][slot], :, p], vp[layer, self.table[s][slot], :, p] = k[x].to(kp.dtype), v[x].to(vp.dtype)
                x += 1
        self.k, self.v = uncanonical(kp, Dh, 0), uncanonical(vp, Dh, 1)

    def attn(self, Dh, layer, seqs, rows, q, window, sinks):
        """(out [rows, heads * Dh], lse [rows, heads]) in 64 bits."""
        kc, vc = canonical(self.k, Dh)[0][layer], canonical(self.v, Dh)[1][layer]
        n_rows, H, _ = q.shape
        Hkv = kc.shape[1]
        out, lse = torch.zeros(n_rows, H, Dh, dtype=torch.float64, device=q.device), torch.full((n_rows, H), -torch.inf, dtype=torch.float64, device=q.device)
        x = 0
        for s, r in zip(seqs, rows):
            for j in range(r):
                at = self.len[s] + j if 0 <= s < self.S else -1
                keys = [k for k in range(at + 1) if (not window or k > at - window or k < sinks) and k // self.P < self.MP and self.table[s][k // self.P] >= 0]
                if keys:
                    pages, pos = torch.tensor([self.table[s][k // self.P] for k in keys], device=q.device), torch.tensor([k % self.P for k in keys], device=q.device)
                    kk = kc[pages, :, pos].double().repeat_interleave(H // Hkv, 1)
                    vv = vc[pages, :, pos].double().repeat_interleave(H // Hkv, 1)
                    score = (kk * q[x].double()).sum(-1) / Dh ** 0.5
                    lse[x] = torch.logsumexp(score, 0)
                    out[x] = (torch.softmax(score, 0)[..., None] * vv).sum(0)
                x += 1
        return out.view(n_rows, -1), lse


def uncanonical(x, Dh, which):
    """The inverse of canonical(): which = 0 K, 1 V."""
    L, N, H, P, _ = x.shape
    flat = x.reshape(L, N, H, P // 32, 32 * Dh)
    ids = torch.arange(32 * Dh, device=x.device).view(1, 1, 1, 1, -1)
    order = canonical(ids, Dh)[which].reshape(-1)
    out = torch.empty_like(flat)
    out[..., order] = flat
    return out
