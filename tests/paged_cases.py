"""More cases of the paged attention: calls whose slots are split, records of chosen coefficients,
and the mean square of the errors that the number formats leave."""
from __future__ import annotations

import numpy as np

import oracle as O
from paged_ref import D, G, MapModel, attention64, codec, default_scale, pack_meta, to_pool

KV = 2

# lens, new tokens, query heads on a KV head (two KV heads): calls whose slots are split
SPLIT = {
    "one": ([2000], [40], 4),
    "last_part_of_129": ([1409], [64], 4),
    "last_part_of_one": ([2305], [5], 4),
    "rows_17": ([2600], [17], 1),
    "seven_heads": ([3000], [70], 7),
    "ragged": ([3000, 90, 700, 0], [40, 30, 1, 0], 4),
    "units_over_parts": ([2600, 2300], [600, 80], 4),
    "long": ([9000, 300], [20, 20], 4),
}


def records_of(codes, z, s, bits, p):
    """Records [n, W] and coefficients [n, 128] in 64 bits from codes [n, 128], zero points and
    scales [n, groups]."""
    z, s = z.astype(np.float16), s.astype(np.float16)
    meta = s.view(np.uint16).astype(np.uint32) | (z.view(np.uint16).astype(np.uint32) << 16)
    live = np.repeat(np.asarray(bits) > 0, G)
    codes = np.where(live, codes, 0).astype(np.uint8)
    coef = np.where(live, np.repeat(z.astype(np.float64), G, 1) + np.repeat(s.astype(np.float64), G, 1) * codes, 0.0)
    return O.pack(codes, pack_meta(meta, bits), bits, p), coef


class Built:
    """A paged cache from functions coefs(b, head, tensor, bits, p, n) -> records, coefficients, with
    queries [n, KV * n_qh, 128] of the given type."""

    def __init__(self, lens, new, n_qh, bits_k, bits_v, words, coefs, query, page=64, seed=0, mean_k=1.0, mean_v=1.0, f32=False):
        import torch
        rng = np.random.default_rng([seed, 23])
        H = len(bits_k)
        self.lens, self.new, self.n_qh, self.H = lens, new, n_qh, H
        (self.ck, pk), (self.cv, pv) = codec(bits_k, words, seed + 1, mean_k), codec(bits_v, words, seed + 2, mean_v)
        need = [-(-n // page) for n in lens]
        ids = rng.permutation(sum(need) + 3)
        m = MapModel(len(ids), page, len(lens), max(need + [1]) + 1)
        pools = [np.full((len(ids), page * H * words), -1, np.int32) for _ in range(2)]
        self.coef = []
        for b, n in enumerate(lens):
            m.table[b, :need[b]] = ids[sum(need[:b]):sum(need[:b + 1])]
            m.lens[b] = n
            per = []
            for h in range(H):
                got = [coefs(b, h, t, (bits_k, bits_v)[t][h], (pk, pv)[t], n) for t in (0, 1)]
                for t in (0, 1):
                    to_pool(pools[t], got[t][0], m.table[b], page, h, H)
                per.append((got[0][1], got[1][1]))
            self.coef.append(per)
        self.pools = [torch.from_numpy(x).cuda() for x in pools]
        self.cache = m.cache()
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        q = torch.from_numpy(query(self).astype(np.float32)).cuda()
        self.q = q if f32 else q.bfloat16()

    def state(self, h):
        return [t.cpu().numpy().astype(np.float64) for t in (self.ck.basis[h], self.ck.mean[h], self.cv.basis[h], self.cv.mean[h])]


def check_split(c, out, lse=None):
    """Every row of case c (as paged_ref's cases) against 64 bits: out of type bfloat16 or float32,
    by element and in the mean square, and the log-sum-exp. Returns the largest |score| reached,
    log2, and the mean square's share of its allowance."""
    import torch
    assert torch.isfinite(out.float()).all()
    got, q = out.float().cpu().numpy().astype(np.float64), c.q.float().cpu().numpy().astype(np.float64)
    bf16 = out.dtype == torch.bfloat16
    at, worst = 0, 0.0
    for b, (L, n) in enumerate(zip(c.lens, c.new)):
        if n == 0:
            continue
        few = n * c.n_qh <= 16
        for h in range(c.H):
            hs = slice(h * c.n_qh, (h + 1) * c.n_qh)
            vk, mk, vv, mv = c.state(h)
            ck, cv = c.coef[b][h]
            want, wlse, swing, most = attention64(q[at:at + n, hs], ck, cv, vk, mk, vv, mv, n, default_scale())
            d = score_error(most, bf16)
            off = got[at:at + n, hs] - want
            tol = element_bound(want, swing, d, L, bf16, few)
            assert (np.abs(off) <= tol).all(), (b, h, float((np.abs(off) / tol).max()))
            if bf16:
                # the expectation by independent roundings, doubled: equal codes of a token's group round alike
                room = 2 * np.sqrt(mean_square(q[at:at + n, hs], ck, cv, vk, vv, mv, n, want).mean())
                rms = np.sqrt((off ** 2).mean())
                worst = max(worst, float(rms / room))
                assert rms <= room, (b, h, float(rms / room))
            if lse is not None:
                g = lse[at:at + n, hs].cpu().numpy().astype(np.float64)
                seen = np.isfinite(wlse)
                assert np.array_equal(np.isneginf(g), ~seen)
                # the sum of weights that are rounded to fp16; the constant q . u, u = scale V m, by 160
                # fp32 steps of at most scale sum |q| |V| |m| in all; the logarithm and its product
                const = default_scale() * np.abs(q[at:at + n, hs]) @ np.abs(vk) @ np.abs(mk)
                size = const + np.abs(np.where(seen, wlse, 0.0)) + most
                lim = d + 2.0 ** -11 * bf16 + (L / 16 + 40) * 2.0 ** -24 + 160 * 2.0 ** -24 * size
                assert (np.abs(g - wlse)[seen] <= lim[seen]).all(), (b, h, float((np.abs(g - wlse)[seen] / lim[seen]).max()))
        at += n
    return worst


def score_error(most, bf16):
    """How far a score may be off (nats) where sum_j |q'_j c_j| is `most`: both factors rounded to
    fp16 (2^-11 each) or to pairs of fp16 parts with the smallest product left out (3 * 2^-22), the
    rotation's bf16 parts (two: 2^-16, three: 2^-22) and 40 fp32 sums; and the exponential's
    argument, of log2 size up to 2 * most + 16, in fp32."""
    f = 2 * 2.0 ** -11 + 2.0 ** -16 if bf16 else 4 * 2.0 ** -22
    return (f + 40 * 2.0 ** -24) * most + 2 * 2.0 ** -24 * (2 * most + 16)


def element_bound(want, swing, d, slots, bf16, few):
    """|error| of an output, where a weight is off by exp(2 d) - 1 (itself and its sum), by its own
    rounding and its sums', and the values and the output rotation by theirs."""
    own = 2 * 2.0 ** -11 if bf16 else (2.0 ** -16 if few else 6 * 2.0 ** -22)
    eps = np.expm1(2 * d)[..., None] * (1 + own) + own + 2.0 ** -11 * bf16 + (slots / 16 + 60) * 2.0 ** -24
    eps = eps + (2.0 ** -15 if bf16 else 2.0 ** -21)
    return eps * swing + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(want) + 1e-30


def mean_square(q, ck, cv, vk, vv, mv, n, want):
    """The expected square of the error of rows q (bfloat16 outputs), averaged over the channels
    [n, heads]: independent roundings of relative mean square 2^-22 / 3 of q', of the coefficients
    and of the weights, to first order; and 2^-16 / 3 of the output's."""
    u = 2.0 ** -22 / 3
    L, scale = len(ck), default_scale()
    got = np.zeros(q.shape[:2])
    for i in range(q.shape[0]):
        see = min(L, max(0, L - n + i + 1))
        if see == 0:
            continue
        k, v = ck[:see], cv[:see]
        qp = scale * q[i] @ vk
        s = qp @ k.T
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        a = p @ v
        for h in range(q.shape[1]):
            away = (v - a[h]) ** 2                                        # [see, 128]
            jac = (k * p[h][:, None]).T @ v - np.outer(p[h] @ k, a[h])     # d a / d q'
            mine = u * (qp[h] ** 2) @ (jac ** 2)
            of_k = u * ((k * qp[h]) ** 2).sum(1) + u                       # of a score, and of the weight itself
            mine = mine + (p[h] ** 2 * of_k) @ away + u * (p[h] ** 2) @ (v ** 2)
            got[i, h] = mine.sum() / D + 2.0 ** -16 / 3 * (want[i, h] ** 2).mean()
    return got
