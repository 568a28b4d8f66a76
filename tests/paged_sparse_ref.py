"""What the tests of drafted trees and of listed blocks compare with: caches of given records, attention over any
set of slots in 64 bits, boxes, block values, and what each kind of call may see."""
from __future__ import annotations

import numpy as np

from paged_cases import Built
from paged_ref import D, G, allowed, default_scale, records

B8 = [[5, 1, 0, 0], [4, 2, 0, 0]]           # 8-word records
ALL = [[8, 7, 6, 5], [1, 2, 3, 4]]          # every width
NONE = [[0, 0, 0, 0], [0, 3, 0, 2]]         # nothing kept; a dropped first group
BLOCK = 64


def cache(lens, new, n_qh=4, bits_k=B8, bits_v=None, words=8, page=64, f32=False, seed=0, scale=1.0, q_scale=2.0):
    """A paged cache of random records, NaN metadata in every slot that no sequence holds."""
    rng = np.random.default_rng([seed, 91])
    bits_v = bits_k[::-1] if bits_v is None else bits_v
    n = sum(new)
    return Built(lens, new, n_qh, bits_k, bits_v, words, lambda b, h, t, bits, p, m: records(bits, p, m, rng, scale),
                 lambda c: q_scale * rng.standard_normal((n, len(bits_k) * n_qh, D)), page=page, seed=seed, f32=f32)


def attend64(q, ck, cv, vk, mk, vv, mv, sees, scale):
    """Rows q [n, heads, 128] of one KV head over the slots that sees [n, L] says, in 64 bits -> out, lse, and
    what paged_ref.allowed takes: the outputs' sum of weighted magnitudes, sum_j |q'_j c_j| at its largest."""
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    swing, most = np.zeros(q.shape), np.zeros(q.shape[:2])
    for i in range(q.shape[0]):
        at = np.flatnonzero(sees[i])
        if not len(at):
            continue
        k, v = ck[at], cv[at]
        qp = scale * q[i] @ vk
        s = qp @ k.T + (qp @ mk)[:, None]
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        lse[i] = (np.log(total) + top)[:, 0]
        p /= total
        chat = p @ v + mv
        out[i] = chat @ vv.T
        swing[i] = (p @ np.abs(v)) @ np.abs(vv).T + np.abs(chat) @ np.abs(vv).T
        most[i] = (np.abs(qp) @ np.abs(k).T).max(1)
    return out, lse, swing, most


def check(c, sees, out, lse=None, ends=None, scale=None):
    """Every row of cache c against 64 bits: sees(b, kv) -> [new tokens, slots]. Returns the largest share of an
    allowance that was used."""
    import torch
    assert torch.isfinite(out.float()).all()
    got, q = out.float().cpu().numpy().astype(np.float64), c.q.float().cpu().numpy().astype(np.float64)
    bf16 = out.dtype == torch.bfloat16
    scale = scale or default_scale()
    at, worst = 0, 0.0
    for b, n in enumerate(c.new):
        for h in range(c.H):
            hs = slice(h * c.n_qh, (h + 1) * c.n_qh)
            vk, mk, vv, mv = c.state(h)
            ck, cv = c.coef[b][h]
            see = sees(b, h)
            slots = max(1, int(see.sum(1).max(initial=0)))
            want, wlse, swing, most = attend64(q[at:at + n, hs], ck, cv, vk, mk, vv, mv, see, scale)
            off, tol = np.abs(got[at:at + n, hs] - want), allowed(want, swing, most, slots, bf16, not bf16)
            assert (off <= tol).all(), (b, h, float((off / np.maximum(tol, 1e-300)).max()))
            worst = max(worst, float((off / np.maximum(tol, 1e-300)).max(initial=0.0)))
            if lse is not None:
                g = lse[at:at + n, hs].cpu().numpy().astype(np.float64)
                seen = np.isfinite(wlse)
                assert np.array_equal(np.isneginf(g), ~seen)
                # the score's error, the rounded weights' sum, and q . u by 160 fp32 steps of at most scale sum |q| |V| |m|
                const = scale * np.abs(q[at:at + n, hs]) @ np.abs(vk) @ np.abs(mk)
                f = 40 * 2.0 ** -24 + (2 * 2.0 ** -11 + 2.0 ** -16 if bf16 else 4 * 2.0 ** -22)
                lim = f * most + 2.0 ** -18 + 2.0 ** -11 * bf16 + (slots / 16 + 40) * 2.0 ** -24
                lim = lim + 160 * 2.0 ** -24 * (const + np.abs(np.where(seen, wlse, 0.0)) + most)
                assert (np.abs(g[seen] - wlse[seen]) <= lim[seen]).all(), (b, h)
        at += n
    return worst


def tree(kind, new, seed=0):
    """Parents of every sequence's new tokens, one after the other."""
    rng = np.random.default_rng([seed, 5])
    got = []
    for n in new:
        i = np.arange(n)
        got.append({"chain": i - 1, "star": np.full(n, -1), "pairs": (i + 1) // 2 - 1,
                    "comb": np.where(i % 2, i - 1, i - 2).clip(-1),
                    "random": np.array([rng.integers(-1, x) for x in i], np.int64)}[kind])
    return np.concatenate(got + [np.zeros(0, np.int64)]).astype(np.int64)


def tree_sees(lens, new, parents):
    """sees(b, kv) of drafted trees; a parent that is no earlier token counts as none."""
    at = np.concatenate([[0], np.cumsum(new)])

    def sees(b, _kv):
        L, n = max(lens[b], 0), new[b]
        past = lens[b] - n
        s = np.zeros((n, L), bool)
        for i in range(n):
            if past + i < 0 or lens[b] < 0:
                continue
            s[i, :max(past, 0)] = True
            j = i
            while j >= 0:
                if past + j >= 0:
                    s[i, past + j] = True
                up = int(parents[at[b] + j])
                j = up if 0 <= up < j else -1
        return s
    return sees


def list_sees(lens, new, blocks):
    """sees(b, kv) of listed blocks [tokens, kv, most]: entries above all before them that the token sees."""
    at = np.concatenate([[0], np.cumsum(new)])

    def sees(b, kv):
        L, n = max(lens[b], 0), new[b]
        s = np.zeros((n, L), bool)
        for i in range(n):
            lim, top = (lens[b] - n + i + 1 if lens[b] >= 0 else 0), -1
            for x in blocks[at[b] + i, kv]:
                if x > top and x * BLOCK < lim:
                    s[i, x * BLOCK:min(lim, (x + 1) * BLOCK)] = True
                top = max(top, x)
        return s
    return sees


def boxes(coef, end):
    """Least and largest coefficients [blocks, 2, 128] over the slots before `end`."""
    n = -(-end // BLOCK)
    return np.stack([[coef[64 * i:min(end, 64 * i + 64)].min(0), coef[64 * i:min(end, 64 * i + 64)].max(0)] for i in range(n)]) \
        if n else np.zeros((0, 2, D))


def box_of(pool, table_row, block, page, kv, n_kv, bits):
    """A block's box [2, 128] out of a box pool (numpy int32), zeros where the group is dropped; and its raw places."""
    tpp = page // 64
    p = pool.reshape(pool.shape[0], n_kv, tpp, 256 // 2).view(np.float16).reshape(pool.shape[0], n_kv, tpp, 4, 2, G)
    raw = p[table_row[block // tpp], kv, block % tpp].astype(np.float64)
    got = np.zeros((2, D))
    for slot, g in enumerate(np.flatnonzero(np.asarray(bits) > 0)):
        got[:, G * g:G * g + G] = raw[slot]
    return got, raw


def block_values(q, box, basis, sees):
    """Values [blocks] of one (token, KV head) in 64 bits, q [heads, 128], box [blocks, 2, 128], -inf for blocks not
    seen; and the largest sum_j |q'_j box_j|, by which values may be off."""
    qp = q @ basis
    s = np.maximum(qp, 0) @ box[:, 1].T + np.minimum(qp, 0) @ box[:, 0].T
    s = np.where(sees, s, -np.inf)
    size = (np.abs(qp) @ np.abs(box).max(1).T).max()
    return (s - s.max(1, keepdims=True)).max(0), size
