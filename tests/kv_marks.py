"""Inputs of the paged cache's attention whose answer names every tile of tokens that went into it.

A token's value is 1 in one column, which its tile of sixteen and its head and sequence choose, and 0 in the others; its weight is a
power of two, which differs between the query heads of a group and, for every other one, grows along the sequence.  So all sums are
exact in fp32 (at most 2^17 tokens with weights from 1 to 2^-6: 23 bits), and what an answer may be off is the division, 2^-23 for the
reciprocal, 2^-24 for each of two products and 2^-23 for each weight's exp2, and its rounding: 2^-20 and half a step.  A column gets a few
dozen tiles: one that is missing, or counted for another head, moves it by percents.
"""
import numpy as np

TILE = 16
LN2 = float(np.float32(np.log(2.0)))  # as the softmax's scale: times log2(e) it is 1 in fp32
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp8": 2.0 ** -8}  # half a step of the outputs


class Marks:
    def __init__(self, dtype, Hq, Hkv, Dk, Dv, page, lens, seed=0):
        self.dtype, self.Hq, self.Hkv, self.Dk, self.Dv, self.page, self.lens = dtype, Hq, Hkv, Dk, Dv, page, list(lens)
        assert max(lens) <= 2 ** 17
        rng = np.random.default_rng(seed)
        per = [-(-n // page) for n in self.lens]
        self.width, self.n_pages = max(per), sum(per) + 1
        order, at = rng.permutation(self.n_pages), 0
        self.table = np.full((len(lens), self.width), 2 ** 30, dtype=np.int32)  # entries behind the last page are never used
        self.k = np.full((self.n_pages, Hkv, page, Dk), np.nan, dtype=np.float32)  # nor rows behind the last token
        self.v = np.full((self.n_pages, Hkv, page, Dv), np.nan, dtype=np.float32)
        self.k_scale = 0.5 if dtype == "fp8" else 1.0
        for b, n in enumerate(self.lens):
            self.table[b, :per[b]] = order[at:at + per[b]]
            at += per[b]
            if n == 0:
                continue
            j = np.arange(n)
            pg, row = self.table[b, j // page], j % page
            for hk in range(Hkv):
                keys, vals = np.zeros((n, Dk), np.float32), np.zeros((n, Dv), np.float32)
                keys[:, 0], keys[:, 1] = self.level(j) / self.k_scale, self.ramp(j, n) / self.k_scale
                vals[j, self.column(b, hk, j)] = 1
                self.k[pg, hk, row], self.v[pg, hk, row] = keys, vals
        h = np.arange(Hq) % (Hq // Hkv)
        self.q = np.zeros((len(lens), Hq, Dk), np.float32)
        self.q[:, :, 0], self.q[:, :, 1] = -(h % 4), h % 2

    @staticmethod
    def level(j):
        return (j.astype(np.uint64) * np.uint64(2654435761) >> np.uint64(13) & np.uint64(1)).astype(np.int64)

    @staticmethod
    def ramp(j, n):
        return 4 * j // n

    def column(self, b, hk, j):
        return (j // TILE + 5 * hk + 3 * b) % self.Dv

    def tokens(self, b, hk, window=0, chosen=None):
        n = self.lens[b]
        if chosen is None:
            return np.arange(max(0, n - window) if window else 0, n)
        j = (np.asarray([c for c in chosen[b][hk] if c >= 0])[:, None] * self.page + np.arange(self.page)).reshape(-1)
        return j[j < n]

    def weights(self, b, g, j):
        return 2.0 ** (-(g % 4) * self.level(j) + g % 2 * self.ramp(j, self.lens[b]))

    def answer(self, b, h, window=0, chosen=None, lost=(), unsummed=(), other=()):
        """(outputs, logarithm) of a query head in 64 bits; of planted mistakes: without the tokens `lost`, with those of `unsummed` in the
        weights' sum but not in the values', with the values of those of `other` weighted by the group's next head."""
        G = self.Hq // self.Hkv
        hk, g = h // G, h % G
        j = self.tokens(b, hk, window, chosen)
        j = j[~np.isin(j, lost)]
        if len(j) == 0:
            return np.zeros(self.Dv), -np.inf
        w, w2 = self.weights(b, g, j), self.weights(b, (g + 1) % G, j)
        u = np.where(np.isin(j, unsummed), 0, np.where(np.isin(j, other), w2 / w2.max() * w.max(), w))
        return np.bincount(self.column(b, hk, j), u, self.Dv) / w.sum(), np.log(w.sum())

    def answers(self, window=0, chosen=None):
        got = [[self.answer(b, h, window, chosen) for h in range(self.Hq)] for b in range(len(self.lens))]
        return np.array([[x[0] for x in row] for row in got]), np.array([[x[1] for x in row] for row in got])

    def wrong(self, out, lse, ref, ref_lse):
        """Where outputs and logarithms are further off than they may be.  A logarithm of up to 20 is a sum of two fp32 numbers, times ln 2: 2^-18."""
        gone = np.isneginf(ref_lse)
        with np.errstate(invalid="ignore"):
            far = np.where(gone, lse != ref_lse, ~(np.abs(lse - ref_lse) <= 2.0 ** -18))
        return ~(np.abs(out - ref) <= (2.0 ** -20 + HALF[self.dtype]) * ref), far
