"""Attention over a paged cache held in 4 bits, where its results are known to a few roundings: every token counts once, and float32
queries and probabilities keep all their bits.  Bounds over sums of thousands of terms, as the other tests have them, leave
room for a token that is lost or counted twice where the work is cut, and for a query in fewer parts."""
import math

import pytest
import torch

from paper_2502_08923_amd import binding as cs
from test_gpu_paged_fp4 import BF, DEV, F32, HALF, U, Cache, gen

pytestmark = pytest.mark.gpu


class Marked(Cache):
    """Streams whose attention counts tokens.  The query is 1 in one feature, where the key of a kept token is 0 and that of a dropped
    one -6 * 2^10: a kept token's score is 0, a dropped one's at most -6144 / 16, which exp makes 0 in float32.  All new tokens are
    kept, so every row sees a kept one.  Values are 1 in one feature, another for the next token (and not the same for
    tokens that are a multiple of 32 apart, where the work is cut, until it comes round), else 0.  So feature f of a row is (kept
    tokens that it sees and that carry f) / (kept tokens that it sees): probabilities are 1, both sums are whole numbers, and so
    are they where partial results are joined (one without a kept token has weight 0)."""

    def __init__(self, lens, rows, KVH, hd, P, dtype=BF, seed=1, **kw):
        super().__init__(lens, rows, KVH, hd, P, dtype, seed, **kw)
        g = gen(seed + 100)
        self.at = hd - 3
        table, self.kept, self.mark = self.table.tolist(), [], []
        heads = torch.arange(KVH, device=DEV)[:, None]
        for b, (L, r) in enumerate(zip(lens, rows)):
            n = L + r
            kept = torch.rand((KVH, n), generator=g, device=DEV) < 0.5
            kept[:, L:] = True
            k = torch.randint(0, 256, (KVH, n, hd // 2), generator=g, dtype=torch.uint8, device=DEV)
            k[..., self.at // 2] = torch.where(kept, 0, 15 << 4 * (self.at % 2)).to(torch.uint8)
            ks = torch.randint(123, 128, (KVH, hd // 32, n), generator=g, dtype=torch.uint8, device=DEV)
            ks[:, self.at // 32] = 137
            t = torch.arange(n, device=DEV)[None]
            mark = (t + 7 * (t // hd) + 5 * heads) % hd
            v = torch.zeros_like(k)
            v.scatter_(2, (mark // 2)[..., None], (2 << 4 * (mark % 2)).to(torch.uint8)[..., None])
            vs = torch.full_like(ks, 127)
            for j in range(-(-n // P)):
                if j not in self.gone[b]:
                    a, e, page = j * P, min(n, (j + 1) * P), table[b][j]
                    for pool, x in ((self.k, k), (self.v, v)):
                        pool[page, :, :e - a] = x[:, a:e]
                    for pool, x in ((self.ks, ks), (self.vs, vs)):
                        pool[page, :, :, :e - a] = x[:, :, a:e]
            for j in self.gone[b]:
                kept[:, j * P:(j + 1) * P] = False
            self.kept.append(kept)
            self.mark.append(mark)

    def counts(self, H, window=0):
        """(kept tokens that carry a feature, kept tokens) of every row's head, float64"""
        carry = torch.zeros((self.ends[-1], H, self.hd), dtype=torch.float64, device=DEV)
        G = H // self.KVH
        for b, (L, r) in enumerate(zip(self.lens, self.rows)):
            if r == 0:
                continue
            one = torch.zeros((self.KVH, L + r + 1, self.hd), dtype=torch.int32, device=DEV)
            one[:, 1:].scatter_(2, self.mark[b][..., None], self.kept[b].int()[..., None])
            upto = one.cumsum(1)
            hi = L + 1 + torch.arange(r, device=DEV)
            lo = (hi - window).clamp(min=0) if window else torch.zeros_like(hi)
            n = (upto[:, hi] - upto[:, lo]).double()                          # [KVH][r][hd]
            carry[self.ends[b]:self.ends[b + 1]] = n.transpose(0, 1).repeat_interleave(G, dim=1)
        return carry, carry.sum(-1, keepdim=True)

    def query(self, H):
        q = torch.zeros((self.R, H, self.hd), dtype=self.dtype, device=DEV)
        q[..., self.at] = 1
        q[self.ends[-1]:] = math.nan
        return q

    def count(self, H, window=0, row0=True, **call):
        """The division and the product with its result are off by 2 u and u at most, a bfloat16 result by half a step more.  A token that
        is lost or counted twice moves its feature by one of as many as carry it, and has to show."""
        q = self.query(H)
        carry, n = self.counts(H, window)
        rel = 3.1 * U + (HALF[BF] if self.dtype == BF else 0)
        assert float(n.min()) > 0 and float(carry.max()) * 2.1 * rel < 1
        got = torch.full_like(q, 9.0)
        cs.cs_paged_fp4_attention(self.pages, q, row0=self.row0 if row0 else None, window=window, out=got, **call)
        live = self.ends[-1]
        want = carry / n
        off = ~((got[:live].double() - want).abs() <= want * rel)
        where = off.nonzero()[:4].tolist()
        assert not where, [(w, float(got[tuple(w)]), float(want[tuple(w)]), float(carry[tuple(w)]), float(n[w[0], w[1], 0])) for w in where]
        assert bool((got[live:] == 9.0).all())


CASES = {
    # few rows: pieces of whole streams, shares of ragged ones, one workgroup per stream over more blocks than its lanes hold pages for
    "singles": dict(lens=[14000, 77, 0, 31, 8192, 8191], rows=[1] * 6),
    "ragged": dict(lens=[9001, 31, 700, 12003, 64, 0, 3333], rows=[4, 1, 3, 2, 0, 1, 4]),
    "blocks": dict(lens=[9000, 10011], rows=[11, 11]),
    "middle": dict(lens=[5000, 40, 2047], rows=[8, 5, 6]),
    "holes": dict(lens=[9500, 700], rows=[2, 3], holes=[(0, 0), (0, 3), (0, 31), (0, 64), (0, 65), (0, 127), (1, 2)]),
    # many rows
    "prompt": dict(lens=[0, 300], rows=[1025, 130]),
    "behind": dict(lens=[4000], rows=[513]),
    "behind_more": dict(lens=[12000, 5], rows=[90, 200]),
    "mixed": dict(lens=[5, 900, 0, 9003, 64, 700, 4001], rows=[0, 1, 513, 1, 2, 2, 1]),
    "holes_many": dict(lens=[7001], rows=[300], holes=[(0, j) for j in (0, 31, 32, 63, 64, 65, 100)]),
}
SHAPES = [(8, 2, 128, 64, "head"), (8, 2, 128, 32, "token"), (4, 4, 128, 32, "both")]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KVH,hd,P,order", SHAPES)
@pytest.mark.parametrize("case", CASES)
def test_every_token_counts_once(case, H, KVH, hd, P, order, dtype):
    c = Marked(KVH=KVH, hd=hd, P=P, dtype=dtype, order=order, pad=2, **CASES[case])
    rows, longest = max(c.rows), max(a + b for a, b in zip(c.lens, c.rows))
    c.count(H, max_rows=rows, max_len=longest)
    c.count(H)                                             # no hints: as long as the table
    c.count(H, max_rows=rows, max_len=16)                  # no cut of the tokens
    c.count(H, max_rows=1, max_len=longest)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KVH,hd", [(7, 1, 64), (4, 1, 256), (6, 2, 96), (5, 5, 160)])
@pytest.mark.parametrize("case", ["singles", "ragged", "blocks", "prompt", "behind", "mixed"])
def test_every_token_counts_once_in_other_heads(case, H, KVH, hd, dtype):
    kw = dict(CASES[case])
    kw["lens"] = [n * hd // 256 for n in kw["lens"]]       # (as many tokens a feature as bfloat16 tells apart)
    c = Marked(KVH=KVH, hd=hd, P=32, dtype=dtype, pad=1, **kw)
    c.count(H, max_rows=max(c.rows), max_len=max(a + b for a, b in zip(c.lens, c.rows)))
    c.count(H, max_rows=max(c.rows), max_len=16)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window", [1, 31, 32, 33, 100, 1024, 9000])
@pytest.mark.parametrize("lens,rows", [([12000, 40, 8200], [1, 1, 1]), ([9000, 50], [11, 4]), ([9007, 3], [90, 300])])
def test_every_token_of_a_window_counts_once(lens, rows, window, dtype):
    c = Marked(lens, rows, 2, 128, 64, dtype, pad=1)
    c.count(8, window=window)
    c.count(8, window=window, max_rows=max(rows), max_len=16)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [63, 64, 65, 130])
def test_every_token_of_many_streams_counts_once(B, dtype):
    """On either side of what a wave's lanes can cut; with and without a block of a prompt among them; equal shares without offsets."""
    lens = [(37 * b * b) % 300 for b in range(B)]
    lens[0], lens[B // 2] = 3500, 2500
    rows = [(b * 7) % 4 for b in range(B)]
    Marked(lens, rows, 1, 64, 32, dtype, pad=2).count(4, max_rows=3, max_len=3503)
    rows[B - 1] = 140
    Marked(lens, rows, 1, 64, 32, dtype, pad=2).count(4, max_rows=140, max_len=3503)
    for each in (1, 2, 30):
        c = Marked(lens, [each] * B, 1, 64, 32, dtype)
        for hint in (0, 16, 3530):
            c.count(4, row0=False, max_len=hint)


def test_every_token_counts_once_behind_a_long_context():
    """As long as bfloat16 tells a token apart: 256 features; and longer in float32."""
    Marked([45000, 30], [1, 1], 1, 256, 64, BF).count(4, max_rows=1, max_len=45001)
    Marked([100001, 70000], [3, 1], 1, 128, 128, F32).count(4, max_rows=3, max_len=100004)
    Marked([65535], [33], 1, 128, 128, F32).count(7, max_rows=33, max_len=65568)


class Pair(Cache):
    """Two tokens of one block share all probability, p = exp(y) and 1 before they are divided by their sum, y the query's first
    feature: their keys are 1 and 0 there, and 0 in the feature where the other tokens have -6 * 2^10 and the query 1 (their
    probability is 0 in float32).  Each carries a 1 in a feature of its own."""

    def __init__(self, lens, rows, KVH, hd, P, **kw):
        super().__init__(lens, rows, KVH, hd, P, F32, **kw)
        table = self.table.tolist()
        for b, (L, r) in enumerate(zip(lens, rows)):
            first = L // 2 & ~31                           # (the pair is in the context: all new rows see it)
            assert L >= 32
            for j in range(-(-(L + r) // P)):
                page = table[b][j]
                self.ks[page], self.vs[page] = 127, 127
                self.ks[page, :, 1] = 137
                self.k[page, :, :, 16] = 15                # feature 32: -6
                self.v[page] = 0
            for t, own in ((first + 3, 0), (first + 20, hd // 2 - 1)):
                page, slot = table[b][t // P], t % P
                self.k[page, :, slot, 16] = 0
                self.k[page, :, slot, 0] = 2 if own == 0 else 0
                self.v[page, :, slot, own] = 2

    def query(self, H, seed):
        """y in -4 .. 4 with all 24 bits of a float32"""
        q = torch.zeros((self.R, H, self.hd), dtype=F32, device=DEV)
        q[..., 0] = torch.rand((self.R, H), generator=gen(seed), device=DEV) * 8 - 4
        q[..., 32] = 1
        return q


@pytest.mark.parametrize("H,KVH,hd,order", [(8, 2, 128, "head"), (8, 2, 128, "token"), (7, 1, 64, "head"), (4, 2, 256, "head"), (3, 3, 96, "both")])
@pytest.mark.parametrize("lens,rows", [([40, 700, 33], [4, 4, 4]), ([3000, 64], [6, 11]), ([9000], [16]), ([700, 100], [90, 300]), ([4000], [160])])
def test_float32_queries_and_probabilities_keep_all_their_bits(lens, rows, H, KVH, hd, order):
    """The scores are y and 0 exactly (y's parts add up without a rounding), with scale 1.  In powers of two they are off by u |x|
    (log2 e) and u |x| more (the differences to the maximum), |x| < 5.8, and the two exp2 by 2 u each: the ratio of the two probabilities by less
    than 0.7 (2 * 5.8 + 1) u + 4 u < 13 u.  Sums of 3 parts of 2 tokens: 6 roundings each for both sums, 2 u each where a
    matrix unit cuts off, 24 u; division and product 3 u: 40 u.  (A query without its third part changes the ratio by up to 256 u,
    a probability without it by up to 128 u.)"""
    c = Pair(lens, rows, KVH, hd, 32, order=order, seed=hd)
    for seed, call in ((1, {}), (2, dict(max_rows=max(rows), max_len=max(a + b for a, b in zip(lens, rows)))), (3, dict(max_rows=max(rows), max_len=16))):
        q = c.query(H, seed)
        got = cs.cs_paged_fp4_attention(c.pages, q, row0=c.row0, scale=1.0, **call).double()
        y = q[..., 0].double()
        for feature, want in ((0, torch.sigmoid(y)), (hd - 2, torch.sigmoid(-y))):
            err = (got[..., feature] - want).abs() / want
            assert bool((err <= 40 * U).all()), float(err.max() / U)
        got[..., 0] = got[..., hd - 2] = 0
        assert bool((got == 0).all())
