"""What the paged cache's tests compare with: the page map as a sequential program over lists,
records made of given codes, attention over the slots in 64 bits, and how far the kernels' number
formats can be off."""
from __future__ import annotations

import math

import numpy as np

import oracle as O
import paper_2608_07915_amd as S

D, G = 128, 32


class MapModel:
    """The page map's rules, one list entry after the other."""

    def __init__(self, n_pages, page, rows, row_pages):
        self.n_pages, self.page, self.rows, self.row_pages = n_pages, page, rows, row_pages
        self.table = np.full((rows, row_pages), -1, np.int64)
        self.lens = np.zeros(rows, np.int64)
        self.refs = np.zeros(n_pages, np.int64)

    def pages(self, n):
        return -(-int(n) // self.page)

    def extend(self, rows, counts):
        """-> ends, copies [(from, to)]."""
        ends, copies, seen, short, lost = [], [], set(), False, []
        for r, c in zip(map(int, rows), map(int, counts)):
            bad = r < 0 or r >= self.rows or r in seen or c < 0
            seen.add(r)
            if bad or self.lens[r] + c > self.row_pages * self.page:
                ends.append(-1)
                continue
            n = int(self.lens[r])
            part = c > 0 and n % self.page != 0
            last = int(self.table[r, n // self.page]) if part else -1
            owners = self.refs[last] - lost.count(last) if part else 0
            shared = part and owners > 1
            start = self.pages(n) - (1 if shared else 0)
            want = self.pages(n + c) - start
            free = np.flatnonzero(self.refs == 0)
            if (short and (want or last in lost)) or want > len(free):
                short = True
                if part:
                    lost.append(last)  # counted on to leave its page
                ends.append(-1)
                continue
            self.table[r, start:start + want] = free[:want]
            self.refs[free[:want]] = 1
            if shared:
                self.refs[last] -= 1
                copies.append((last, int(free[0])))
            self.lens[r] = n + c
            ends.append(n + c)
        return ends, copies

    def fork(self, parents, children):
        ends = []
        for i, (p, c) in enumerate(zip(map(int, parents), map(int, children))):
            ok = 0 <= p < self.rows and 0 <= c < self.rows and c not in list(children[:i]) and p not in list(children)
            if not ok or self.lens[c] != 0:
                ends.append(-1)
                continue
            n = self.pages(self.lens[p])
            self.table[c, :n] = self.table[p, :n]
            np.add.at(self.refs, self.table[p, :n], 1)
            self.lens[c] = self.lens[p]
            ends.append(int(self.lens[p]))
        return ends

    def truncate(self, rows, keep=None):
        for i, r in enumerate(map(int, rows)):
            if not 0 <= r < self.rows:
                continue
            k = 0 if keep is None else max(0, int(keep[i]))
            if k >= self.lens[r]:
                continue
            a, b = self.pages(k), self.pages(self.lens[r])
            np.add.at(self.refs, self.table[r, a:b], -1)
            self.table[r, a:b] = -1
            self.lens[r] = k

    def compact(self):
        used = np.flatnonzero(self.refs > 0)
        n = len(used)
        src, dst = used[used >= n], np.flatnonzero(self.refs[:n] == 0)
        moved = np.arange(self.n_pages + 1)
        moved[src] = dst
        moved[-1] = n
        for r in range(self.rows):
            k = self.pages(self.lens[r])
            self.table[r, :k] = moved[self.table[r, :k]]
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        return moved, list(zip(src.tolist(), dst.tolist()))

    def cache(self):
        import torch
        c = S.PagedCache(self.n_pages, self.page, self.rows, self.row_pages)
        c.table.copy_(torch.from_numpy(self.table))
        c.lens.copy_(torch.from_numpy(self.lens))
        c.refs.copy_(torch.from_numpy(self.refs))
        return c

    def check(self, cache):
        """The device's map holds what this one holds."""
        assert np.array_equal(cache.lens.cpu().numpy(), self.lens)
        assert np.array_equal(cache.refs.cpu().numpy(), self.refs)
        t = cache.table.cpu().numpy()
        for r in range(self.rows):
            k = self.pages(self.lens[r])
            assert np.array_equal(t[r, :k], self.table[r, :k]), r


def codec(bits, words, seed, mean=1.0, device="cuda"):
    """A codec of len(bits) KV heads with the given group widths per head: random orthonormal
    bases and means; records of `words` words."""
    import torch
    rng = np.random.default_rng(seed)
    p = O.Params(budget_bits=32 * words)
    c = S.Codec(S.Params(budget_bits=32 * words), len(bits), device=device)
    for h, b in enumerate(bits):
        q, _ = np.linalg.qr(rng.standard_normal((D, D)))
        c.basis[h] = torch.from_numpy(q.astype(np.float32))
        c.mean[h] = torch.from_numpy((mean * rng.standard_normal(D)).astype(np.float32))
        c.bits[h] = torch.tensor(b, dtype=torch.uint8)
    c.var.fill_(1.0)
    return c, p


def records(bits, p, n, rng, scale=1.0):
    """n records of one head -> words [n, W] and coefficients [n, 128] in 64 bits."""
    codes = np.stack([rng.integers(0, 2 ** int(b), (n, G)) for b in bits], 1).reshape(n, D)
    nG = D // G
    z = (scale * rng.standard_normal((n, nG)) * 2).astype(np.float16)
    s = (scale * rng.uniform(0.2, 1.0, (n, nG)) * 4 / np.maximum(1, 2.0 ** np.asarray(bits) - 1)).astype(np.float16)
    meta = s.view(np.uint16).astype(np.uint32) | (z.view(np.uint16).astype(np.uint32) << 16)
    live = np.repeat(np.asarray(bits) > 0, G)
    codes = np.where(live, codes, 0).astype(np.uint8)
    coef = np.where(live, np.repeat(z.astype(np.float64), G, 1) + np.repeat(s.astype(np.float64), G, 1) * codes, 0.0)
    return O.pack(codes, pack_meta(meta, bits), bits, p), coef


def pack_meta(meta, bits):
    """Metadata [n, groups], zero for dropped groups."""
    return np.where(np.asarray(bits) > 0, meta, 0).astype(np.uint32)


def to_pool(pool, rec, table_row, page, kv, n_kv):
    """Writes records rec [n, W] of one head into the slots 0 .. n of a row of pages (numpy pool
    [n_pages, words of a page])."""
    n, W = rec.shape
    p = pool.reshape(pool.shape[0], n_kv, page // 64, W, 64)
    t = np.arange(n)
    for w in range(W):
        p[table_row[t // page], kv, (t % page) // 64, w, t % 64] = rec[:, w].astype(np.uint32).view(np.int32)


def from_pool(pool, table_row, n, page, kv, n_kv, W):
    p = pool.reshape(pool.shape[0], n_kv, page // 64, W, 64)
    t = np.arange(n)
    return np.stack([p[table_row[t // page], kv, (t % page) // 64, w, t % 64] for w in range(W)], 1).view(np.uint32)


def attention64(q, ck, cv, vk, mk, vv, mv, n, scale):
    """Rows q [n, heads, 128] of the last n of len(ck) slots of one KV head, everything in 64
    bits -> out, lse, and per output |error| / eps if every weight had a relative error of eps:
    sum_j (sum_t p |c_V|)_j |V_ij| + sum_j |chat_j V_ij|, and sum_j |q'_j c_j| at its largest."""
    L = len(ck)
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    swing, most = np.zeros(q.shape), np.zeros(q.shape[:2])
    for i in range(q.shape[0]):
        see = min(L, max(0, L - n + i + 1))
        if see == 0:
            continue
        qp = scale * q[i] @ vk                                   # [heads, 128]
        s = qp @ ck[:see].T + (qp @ mk)[:, None]
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        lse[i] = (np.log(total) + top)[:, 0]
        p /= total
        chat = p @ cv[:see] + mv
        out[i] = chat @ vv.T
        swing[i] = (p @ np.abs(cv[:see])) @ np.abs(vv).T + np.abs(chat) @ np.abs(vv).T
        most[i] = (np.abs(qp) @ np.abs(ck[:see]).T).max(1)
    return out, lse, swing, most


def allowed(out, swing, most, slots, out_bf16, precise):
    """How far an output may be off, element by element.

    A score is a sum of at most 128 products of rounded factors: it is off by at most d = f *
    `most`, where f = 2 * 2^-11 for single fp16 factors, and 3 * 2^-22 for pairs of fp16 parts
    (two roundings and the product left out), plus the fp32 sums' 40 roundings of 2^-24 (24 steps
    of the query's rotation, 16 of the product). Softmax weights are off by exp(2 d) - 1 <= 2.1 d
    (both the weight and its sum), by 2^-21 of the exponential (its argument's rounding: scores up
    to 2^5 in log2 units hold 2^-19 absolute, weighed like d), and by their own rounding; the values
    likewise; the sums over slots take slots / 16 steps of 2^-24 at the worst. The rotation's bf16
    parts leave 2^-15 (two) or 2^-22 (three)."""
    f = 40 * 2.0 ** -24 + (3 * 2.0 ** -22 if precise else 2 * 2.0 ** -11)
    d = (f * most + 2.0 ** -18)[..., None]
    eps = 2.1 * d + (6 * 2.0 ** -22 if precise else 2 * 2.0 ** -11) + (slots / 16 + 40) * 2.0 ** -24
    eps = eps + (2.0 ** -21 if precise else 2.0 ** -15)
    return eps * swing + (2.0 ** -8 * np.abs(out) if out_bf16 else 2.0 ** -24 * np.abs(out)) + 1e-30


def default_scale():
    return 1.0 / math.sqrt(D)
