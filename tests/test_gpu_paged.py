"""The operators of a paged cache against their definitions in float64: norms of query and key heads with the rotary
embedding, append of ragged rows to pages, attention of a chunk of rows over pages.

Tolerances.  u = 2^-24 is half a step of float32, and a value rounded to bfloat16 is off by at most 2^-8 of itself.
Sums of n products in float32 are off by at most n * u of the sum of their magnitudes, whatever their order."""
import math

import pytest
import torch

from paper_2502_08923_amd import binding as cs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(shape, g, dtype, spread=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * spread).to(dtype)


def inv_freq_of(rot, theta=10000.0):
    return torch.tensor([theta ** (-2.0 * j / rot) for j in range(rot // 2)], dtype=torch.float64, device=DEV)


# ------------------------------------------------------------------------------------------------------
# norms and rotation
# ------------------------------------------------------------------------------------------------------

def ref_norm_rope(x, gain, pos, inv_freq, eps):
    """(values, bound on their float32 error before the last rounding), float64"""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    hd = x.shape[-1]
    # the sum of squares is off by hd * u of itself, its root by half of that; root, quotient, products: 6 more roundings
    rel = (hd / 2 + 6) * U if gain is not None else 0.0
    bound = x.abs() * rel
    if inv_freq is not None:
        n = inv_freq.numel()
        a = pos.double()[:, None] * inv_freq[None]
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        lo, hi = x[..., :n].clone(), x[..., n:2 * n].clone()
        y = x.clone()
        y[..., :n], y[..., n:2 * n] = lo * c - hi * s, hi * c + lo * s
        # cosine and sine: the reduced angle is rounded to float32 (at most pi/4: 0.8 u), Taylor's series 4 roundings and
        # 0.03 u dropped; the two products and their sum 2 more of either term
        both = (lo.abs() + hi.abs()) * (rel + 7 * U)
        bound = torch.cat([both, both, bound[..., 2 * n:]], -1)
        x = y
    return x, bound


@pytest.mark.parametrize("tin,tout", [(BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("R,H,KVH,hd,rot", [(1, 1, 1, 8, 8), (1, 32, 8, 128, 128), (3, 28, 4, 128, 128), (88, 32, 8, 128, 64),
                                            (1030, 5, 1, 64, 64), (2, 7, 3, 72, 72), (1025, 3, 2, 80, 32), (5, 4, 4, 256, 256),
                                            (6, 2, 2, 40, 16), (4, 3, 0, 96, 96), (7, 2, 1, 248, 8)])
def test_norm_rope(R, H, KVH, hd, rot, tin, tout):
    g = gen(R * 1000 + hd)
    qkv = randn((R, H + 2 * KVH, hd), g, tin)
    q, k = qkv[:, :H], qkv[:, H:H + KVH] if KVH else None
    pos = torch.randint(0, 200000, (R,), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = 0
    pos[-1] = 2 ** 20 - 1
    f = inv_freq_of(rot)
    qg, kg = 1 + 0.1 * randn((hd,), g, F32), 1 + 0.1 * randn((hd,), g, F32)
    for gains, freq in (((qg, kg), f), ((None, kg), f), ((qg, kg), None), ((None, None), f)):
        qo, ko = cs.cs_op_qk_norm_rope(q, k, pos, freq, *gains, eps=1e-5, out_dtype=tout)
        for x, gain, y in ((q, gains[0], qo), (k, gains[1], ko)):
            if x is None:
                assert y is None
                continue
            want, bound = ref_norm_rope(x, gain, pos, freq, 1e-5)
            assert y.dtype == tout and y.shape == x.shape
            tol = bound * (1 + HALF[tout]) + want.abs() * HALF[tout] + 1e-38
            assert bool(((y.double() - want).abs() <= tol).all()), float(((y.double() - want).abs() - tol).max())


def test_norm_rope_in_place_and_into_strided_rows():
    g = gen(5)
    qkv = randn((37, 40, 128), g, BF)
    pos = torch.arange(37, device=DEV, dtype=torch.int32) * 1000
    gain, f = 1 + 0.1 * randn((128,), g, F32), inv_freq_of(128)
    want = cs.cs_op_qk_norm_rope(qkv[:, :32], qkv[:, 32:36], pos, f, gain, gain)
    wide = torch.full((37, 2, 40, 136), 7.0, dtype=BF, device=DEV)
    out = (wide[:, 0, :32, :128], wide[:, 0, 32:36, :128])
    cs.cs_op_qk_norm_rope(qkv[:, :32], qkv[:, 32:36], pos, f, gain, gain, out=out)
    keep = qkv.clone()
    cs.cs_op_qk_norm_rope(qkv[:, :32], qkv[:, 32:36], pos, f, gain, gain, out=(qkv[:, :32], qkv[:, 32:36]))
    for a, b, c in zip(want, out, (qkv[:, :32], qkv[:, 32:36])):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert torch.equal(qkv[:, 36:], keep[:, 36:])
    wide[:, 0, :36, :128] = 7.0
    assert bool((wide == 7.0).all())


def test_rotation_keeps_far_positions_apart():
    """Positions up to 2^31 - 1: the angle is exact to 2^-20 turns there (float64 keeps 2^-53 of 2^31 turns / 6.28)."""
    pos = torch.tensor([0, 1, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1, -5], dtype=torch.int32, device=DEV)
    f = inv_freq_of(64)
    x = torch.zeros((6, 1, 64), device=DEV)
    x[:, :, :32] = 1.0
    y, _ = cs.cs_op_qk_norm_rope(x, None, pos, f)
    a = pos.double()[:, None] * f[None]
    # two roundings of 2^-53 relative in the number of turns on either side
    tol = 7 * U + 4 * a.abs() * 2.0 ** -53
    assert bool(((y[:, 0, :32].double() - torch.cos(a)).abs() <= tol).all())
    assert bool(((y[:, 0, 32:].double() - torch.sin(a)).abs() <= tol).all())


# ------------------------------------------------------------------------------------------------------
# a paged cache whose dead places are poisoned
# ------------------------------------------------------------------------------------------------------

class Cache:
    """Pools, table and lengths of ragged streams; everything that no live token owns is NaN, and table entries behind a
    stream's last page are out of range."""

    def __init__(self, lens, rows, KVH, hd, P, dtype, seed=1, order="head", pad=0, holes=(), spare=2, shared=0):
        g = gen(seed)
        B = len(lens)
        self.lens, self.rows, self.P, self.pad = list(lens), list(rows), P, pad
        need = [-(-(n + r) // P) for n, r in zip(lens, rows)]
        total = sum(need) + spare
        shape = {"head": (total, KVH, P, hd), "token": (total, P, KVH, hd), "both": (total, KVH, P, 2, hd + 8)}[order]
        if order == "both":                              # keys and values of a token side by side, padded rows
            pool = torch.full(shape, math.nan, dtype=dtype, device=DEV)
            self.k, self.v = pool[..., 0, :hd], pool[..., 1, :hd]
        else:
            self.k, self.v = (torch.full(shape, math.nan, dtype=dtype, device=DEV) for _ in range(2))
            if order == "token":
                self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        names = torch.randperm(total, generator=g, device=DEV).tolist()
        width = max(need + [1]) + 1
        table = [[(-1, 1 << 30, -2 ** 31)[j % 3] for j in range(width)] for _ in range(B)]
        for b in range(B):
            for j in range(need[b]):
                table[b][j] = table[0][j] if b and j < shared else names.pop()
        self.k_tok, self.v_tok = [], []                  # [KVH][n][hd] of every stream
        for b in range(B):
            n = lens[b] + rows[b]
            kt, vt = randn((KVH, n, hd), g, dtype), randn((KVH, n, hd), g, dtype)
            if b and shared:
                m = min(n, shared * P)
                kt[:, :m], vt[:, :m] = self.k_tok[0][:, :m], self.v_tok[0][:, :m]
            self.k_tok.append(kt)
            self.v_tok.append(vt)
            for j in range(need[b]):
                a, e = j * P, min(n, (j + 1) * P)
                self.k[table[b][j], :, :e - a] = kt[:, a:e]
                self.v[table[b][j], :, :e - a] = vt[:, a:e]
        self.gone = [set() for _ in range(B)]
        for b, j in holes:                               # evicted pages: poisoned, the table names nothing
            self.k[table[b][j]] = math.nan
            self.v[table[b][j]] = math.nan
            table[b][j] = (-1, total, 2 ** 31 - 1)[j % 3]
            self.gone[b].add(j)
        self.table = torch.tensor(table, dtype=torch.int32, device=DEV)
        self.length = torch.tensor(lens, dtype=torch.int32, device=DEV)
        ends = [0]
        for r in rows:
            ends.append(ends[-1] + r)
        self.ends = ends
        self.R = ends[-1] + pad
        self.row0 = torch.tensor(ends, dtype=torch.int32, device=DEV)
        self.pages = cs.Pages(self.k, self.v, self.table, self.length)

    def reference(self, q, scale, window=0):
        """(out, sum of p|v|, bound on the error of a score) in float64, rows behind the last stream 0"""
        KVH, hd = self.k.shape[1], self.k.shape[3]
        H = q.shape[1]
        G = H // KVH
        out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
        mag, delta = torch.zeros_like(out), torch.zeros(q.shape[:2] + (1,), dtype=torch.float64, device=DEV)
        for b, (L, r) in enumerate(zip(self.lens, self.rows)):
            if r == 0:
                continue
            n = L + r
            k, v = self.k_tok[b].double(), self.v_tok[b].double()
            t = torch.arange(n, device=DEV)
            at = L + torch.arange(r, device=DEV)
            sees = t[None] <= at[:, None]
            if window:
                sees &= t[None] > at[:, None] - window
            for j in self.gone[b]:
                sees[:, j * self.P:(j + 1) * self.P] = False
            for g in range(KVH):
                for u in range(G):
                    x = q[self.ends[b]:self.ends[b] + r, g * G + u].double()
                    s = (x @ k[g].T.contiguous()) * scale
                    d = (x.abs() @ k[g].abs().T.contiguous()) * scale
                    d = torch.where(sees, d, torch.zeros_like(d)).amax(1)
                    s = s.masked_fill(~sees, -math.inf)
                    m = s.amax(1, keepdim=True)
                    p = torch.where(sees, torch.exp(s - torch.where(m.isinf(), torch.zeros_like(m), m)), torch.zeros_like(s))
                    l = p.sum(1, keepdim=True)
                    p = torch.where(l > 0, p / l, p)
                    rows = slice(self.ends[b], self.ends[b] + r)
                    out[rows, g * G + u] = p @ v[g]
                    mag[rows, g * G + u] = p @ v[g].abs()
                    delta[rows, g * G + u, 0] = d
        return out, mag, delta

    def check(self, H, window=0, scale=None, seed=3, spread=2.0, **call):
        KVH, hd = self.k.shape[1], self.k.shape[3]
        q = randn((self.R, H, hd), gen(seed), self.k.dtype, spread)
        scale_v = 1 / math.sqrt(hd) if scale is None else scale
        want, mag, delta = self.reference(q, scale_v, window)
        if self.pad:
            q[self.ends[-1]:] = math.nan
        out = torch.full_like(q, 123.0)
        got = cs.cs_paged_attention(self.pages, q, row0=self.row0, window=window, scale=scale, out=out, **call)
        assert got is out
        live = self.ends[-1]
        assert bool((got[live:] == 123.0).all()), "rows behind the last stream were written"
        self.close(got[:live], want[:live], mag[:live], delta[:live], hd)
        return q, got

    def close(self, got, want, mag, delta, hd):
        """A score is off by (hd + 4) * u of sum |q_d k_d| * scale (products, sums, the scale and the exponent's subtraction)
        and exp2 by 2 u more; a probability by as much, relatively, and the result by twice that of sum p|v| (numerator and
        denominator).  Sums over n tokens and the joins: (n + 16) u.  bfloat16: the probabilities are rounded, numerator and
        denominator alike, 2 * 2^-8 together, and the result once."""
        n = max(a + b for a, b in zip(self.lens, self.rows))
        rel = 2 * ((hd + 4) * delta + 2) * U + 2 * (n + 16) * U
        if got.dtype == BF:
            rel = rel + 2 * HALF[BF]
        tol = mag * rel + want.abs() * HALF[got.dtype] + 1e-30
        err = (got.double() - want).abs()
        assert bool((err <= tol).all()), (float((err - tol).max()), int((~(err <= tol)).sum()), err.shape)


SHAPES = [(4, 4, 64), (8, 2, 128), (7, 1, 128), (3, 3, 8), (6, 2, 72), (16, 1, 256), (5, 5, 40), (4, 1, 96), (12, 4, 200)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KVH,hd", SHAPES)
@pytest.mark.parametrize("P", [16, 64])
def test_attention_shapes(H, KVH, hd, P, dtype):
    lens, rows = [0, 1, 15, 16, 17, 63, 200, 129], [1, 1, 3, 1, 0, 2, 11, 5]
    Cache(lens, rows, KVH, hd, P, dtype, seed=hd, order="token" if P == 16 else "head", pad=3).check(H)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("P", [16, 32, 128, 1024])
@pytest.mark.parametrize("rows", [1, 4, 11, 13, 33, 70, 150, 300])
def test_attention_equal_rows(rows, P, dtype):
    lens = [0, 31, 257, 1100]
    c = Cache(lens, [rows] * 4, 2, 128, P, dtype, seed=rows)
    q, got = c.check(8)
    again = cs.cs_paged_attention(c.pages, q, max_rows=rows, max_len=1100 + rows)
    assert torch.equal(got, again) or bool(((got.double() - again.double()).abs() <= 2.0 ** -6).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window", [1, 2, 16, 33, 100, 5000])
@pytest.mark.parametrize("rows", [1, 9, 130])
def test_attention_window(rows, window, dtype):
    Cache([0, 40, 700, 1500], [rows, rows, 0, rows], 2, 64, 16, dtype, seed=window).check(4, window=window)
    Cache([0, 40, 700, 1500], [rows, rows, 0, rows], 1, 128, 32, dtype, seed=window).check(3, window=window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 11, 70, 150])
@pytest.mark.parametrize("window", [1, 20, 33, 100])
def test_attention_behind_the_window_anything(window, rows, dtype):
    """Tokens that no new row's window reaches any more may hold NaN or infinities."""
    for hd, P in ((64, 16), (128, 64)):
        c = Cache([30, 333, 64], [rows] * 3, 2, hd, P, dtype, seed=window)
        table = c.table.cpu()
        for b, n in enumerate(c.lens):
            for t in range(max(0, n - window + 1)):
                c.k[int(table[b][t // P]), :, t % P] = (math.nan, math.inf, -math.inf)[t % 3]
                c.v[int(table[b][t // P]), :, t % P] = (math.inf, math.nan, -math.inf)[t % 3]
        c.check(4, window=window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 6, 100])
@pytest.mark.parametrize("P", [16, 32, 64])
def test_attention_evicted_pages(P, rows, dtype):
    """Pages that the table no longer names are not attended to, whatever lies in them; a row that sees nothing else is 0."""
    lens = [3 * P, 10 * P + 5, P - 1]
    holes = [(0, 0), (0, 2), (1, 1), (1, 5), (1, 6), (1, 7)]
    c = Cache(lens, [rows] * 3, 2, 64, P, dtype, seed=P, holes=holes)
    c.check(4)
    if rows == 1:
        c = Cache([P - 1, 2 * P], [1, 1], 2, 64, P, dtype, seed=P, holes=[(0, 0)])
        _, got = c.check(4)
        assert bool((got[0] == 0).all())
        c = Cache([4 * P - 1], [1], 2, 64, P, dtype, seed=P, holes=[(0, 3)])
        _, got = c.check(4, window=P // 2)
        assert bool((got[0] == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_shared_prefix_and_interleaved_pool(dtype):
    Cache([150, 200, 133], [4, 1, 40], 2, 64, 32, dtype, order="both", shared=4).check(8)
    Cache([150, 200, 133], [4, 1, 2], 2, 128, 16, dtype, order="both", shared=8).check(2)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_mixed_batch(dtype):
    """A prompt block next to single tokens, streams without rows at both ends, hints that are right, absent and wrong."""
    lens, rows = [5, 900, 0, 3000, 64, 700, 0], [0, 1, 513, 1, 1, 2, 0]
    c = Cache(lens, rows, 2, 128, 32, dtype, pad=5, seed=9)
    for hints in ({}, dict(max_rows=513, max_len=3001), dict(max_rows=1, max_len=16), dict(max_rows=4096, max_len=100000)):
        c.check(8, **hints)


@pytest.mark.parametrize("dtype,rows,lens", [(BF, 1, [30000, 77]), (BF, 11, [9000, 20011]), (BF, 40, [12345]), (F32, 1, [20000]),
                                             (F32, 7, [6000, 100]), (BF, 513, [4000]), (BF, 1025, [0])])
def test_attention_long_contexts(dtype, rows, lens):
    c = Cache(lens, [rows] * len(lens), 2, 128, 64, dtype, seed=rows)
    c.check(8)
    c.check(8, max_rows=rows, max_len=max(lens) + rows)


@pytest.mark.parametrize("hd,H,KVH", [(128, 8, 2), (64, 4, 4), (256, 4, 2), (96, 6, 1)])
@pytest.mark.parametrize("lens,rows", [([0], [985]), ([0, 300], [130, 700]), ([2000, 0, 70], [200, 49, 1]), ([8000], [90])])
def test_attention_prompt_blocks(lens, rows, hd, H, KVH):
    """Prompt blocks on empty and on filled caches, alone and ragged: tiles of 128 and of 256 query rows."""
    c = Cache(lens, rows, KVH, hd, 32, BF, seed=hd, pad=2)
    c.check(H)
    c.check(H, max_rows=max(rows), max_len=max(a + b for a, b in zip(lens, rows)))
    c.check(H, window=100)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,lens,window", [(1, [30000, 50], 0), (40, [9000], 0), (70, [9000, 9], 0), (300, [7001], 0), (2, [20000], 9000),
                                              (90, [12000], 5000)])
def test_attention_one_range_over_a_long_context(rows, lens, window, dtype):
    """A hint of short contexts leaves one workgroup a whole one: more blocks than its lanes hold page numbers for."""
    holes = [(0, j) for j in (0, 63, 64, 65, 127, 128, 200)]
    Cache(lens, [rows] * len(lens), 1, 64, 16, dtype, seed=rows, holes=holes).check(2, max_rows=rows, max_len=16, window=window)
    Cache(lens, [rows] * len(lens), 1, 128, 32, dtype, seed=rows).check(3, max_rows=rows, max_len=16, window=window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [2, 63, 64, 65, 130])
def test_attention_many_ragged_streams(B, dtype):
    """Lengths and rows of every size, on either side of what a wave's lanes can cut; two streams carry most of the tokens."""
    lens = [(37 * b * b) % 90 for b in range(B)]
    lens[0], lens[B // 2 if B > 2 else 1] = 5000, 2500
    rows = [(b * 7) % 5 for b in range(B)]
    rows[0] = 3
    Cache(lens, rows, 1, 64, 16, dtype, seed=B, pad=2).check(4)
    rows[B - 1] = 140                                     # one prompt block among them
    Cache(lens, rows, 1, 64, 16, dtype, seed=B, pad=2).check(4, max_rows=140, max_len=5003)
    c = Cache(lens, [2] * B, 1, 64, 32, dtype, seed=B)
    c.check(4, max_rows=2, max_len=5003, window=700)
    q = randn((2 * B, 4, 64), gen(5), dtype)              # equal shares without offsets, one range and several
    c.close(cs.cs_paged_attention(c.pages, q, max_len=16), *c.reference(q, 0.125), 64)
    c.close(cs.cs_paged_attention(c.pages, q, max_len=5003), *c.reference(q, 0.125), 64)
    c = Cache(lens, [30] * B, 1, 64, 32, dtype, seed=B)
    q = randn((30 * B, 4, 64), gen(5), dtype)
    c.close(cs.cs_paged_attention(c.pages, q, max_len=16), *c.reference(q, 0.125), 64)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_scale_and_peaked_scores(dtype):
    c = Cache([300, 1], [5, 2], 2, 64, 16, dtype)
    c.check(4, scale=0.01)
    c.check(4, spread=30.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_lengths_outside_the_table(dtype):
    """Negative lengths count as 0; tokens that the table has no column for do not exist."""
    c = Cache([20, 40], [1, 1], 2, 64, 16, dtype)
    q = randn((2, 4, 64), gen(1), dtype)
    want = cs.cs_paged_attention(c.pages, q)
    short = cs.Pages(c.k, c.v, c.table[:, :2].contiguous(), c.length)
    c.length.copy_(torch.tensor([-7, 2 ** 31 - 1]))
    got = cs.cs_paged_attention(short, q)
    c.length.copy_(torch.tensor([0, 31]))
    assert torch.equal(got, cs.cs_paged_attention(c.pages, q))
    assert not torch.equal(got, want)


def test_attention_row_offsets_that_make_no_sense():
    """Offsets outside 0..R or decreasing leave rows out; nothing outside the tensors is touched."""
    c = Cache([20, 40, 10], [2, 2, 2], 2, 64, 16, BF)
    q = randn((6, 4, 64), gen(1), BF)
    out = torch.full_like(q, 5.0)
    for bad in ([0, 100, 3, 6], [-50, 2, 2000000000, 6], [6, 4, 2, 0], [0, -1, -2, -3], [2 ** 31 - 1] * 4):
        row0 = torch.tensor(bad, dtype=torch.int32, device=DEV)
        cs.cs_paged_attention(c.pages, q, row0=row0, out=out)
        cs.cs_paged_append(c.pages, q[:, :2].contiguous(), q[:, :2].contiguous(), row0=row0)
    c = Cache([3000, 40, 1000] + [9] * 70, [2] * 73, 1, 64, 16, BF)        # with token ranges, and more streams than a wave has lanes
    q = randn((146, 2, 64), gen(1), BF)
    for n in (3, 73):
        p = cs.Pages(c.k, c.v, c.table[:n], c.length[:n])
        for bad in ([0, 146] * 37, [146 - 2 * b for b in range(74)], [0] * 73 + [146], [(b * 97) % 300 - 50 for b in range(74)]):
            cs.cs_paged_attention(p, q, row0=torch.tensor(bad[:n + 1], dtype=torch.int32, device=DEV), max_rows=2, max_len=3002)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_strided_rows_and_in_place(dtype):
    c = Cache([100, 3], [5, 5], 2, 64, 16, dtype)
    q = randn((10, 4, 64), gen(4), dtype)
    want = cs.cs_paged_attention(c.pages, q)
    wide = torch.full((10, 3, 8, 72), 9.0, dtype=dtype, device=DEV)
    src, dst = wide[:, 0, :4, :64], wide[:, 2, 4:, :64]
    src.copy_(q)
    cs.cs_paged_attention(c.pages, src, out=dst)
    assert torch.equal(dst, want)
    assert bool((wide[:, 1] == 9.0).all()) and bool((wide[..., 64:] == 9.0).all()) and torch.equal(src, q)
    cs.cs_paged_attention(c.pages, src, out=src)
    assert torch.equal(src, want)
    turned = q.permute(1, 0, 2).contiguous().permute(1, 0, 2)         # head-major rows
    assert torch.equal(cs.cs_paged_attention(c.pages, turned), want)


# ------------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tin,dtype", [(BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("order", ["head", "token", "both"])
@pytest.mark.parametrize("KVH,hd,rot,P", [(8, 128, 128, 64), (1, 64, 64, 16), (3, 72, 72, 32), (4, 80, 32, 16), (2, 256, 0, 128), (5, 8, 8, 16)])
def test_append(KVH, hd, rot, P, order, tin, dtype):
    lens, rows = [0, 5, 16, 15, 31, 0, 1000], [17, 1, 0, 3, 33, 0, 40]
    c = Cache(lens, rows, KVH, hd, P, dtype, order=order, pad=4, seed=hd + P, holes=[(4, 1)] if P == 32 else ())
    g = gen(77)
    kv = randn((c.R, 2 * KVH, hd), g, tin)
    kv[c.ends[-1]:] = math.nan
    k, v = kv[:, :KVH], kv[:, KVH:]
    f = inv_freq_of(rot) if rot else None
    k_pool, v_pool = c.k.clone(), c.v.clone()
    cs.cs_paged_append(c.pages, k, v, row0=c.row0, inv_freq=f)
    torch.cuda.synchronize()
    table = c.table.cpu()
    touched = torch.zeros((c.k.shape[0], P), dtype=torch.bool, device=DEV)
    for b, (L, r) in enumerate(zip(lens, rows)):
        pos = torch.arange(L, L + r, device=DEV, dtype=torch.int32)
        want, bound = ref_norm_rope(k[c.ends[b]:c.ends[b] + r], None, pos, f, 0.0)
        for i in range(r):
            at = L + i
            if at // P in c.gone[b]:
                continue
            page, slot = int(table[b][at // P]), at % P
            touched[page, slot] = True
            tol = bound[i] * (1 + HALF[dtype]) + want[i].abs() * HALF[dtype]
            assert bool(((c.k[page, :, slot].double() - want[i]).abs() <= tol).all()), (b, i)
            assert torch.equal(c.v[page, :, slot], v[c.ends[b] + i].to(dtype)), (b, i)
    rest = ~touched
    for new, old in ((c.k, k_pool), (c.v, v_pool)):
        a, b = new.permute(0, 2, 1, 3)[rest], old.permute(0, 2, 1, 3)[rest]
        assert torch.equal(torch.nan_to_num(a.float(), nan=1e30), torch.nan_to_num(b.float(), nan=1e30)), "a slot nobody owns was written"


def test_append_past_the_table_and_equal_shares():
    c = Cache([28, 40], [3, 3], 2, 64, 16, BF)
    k = randn((6, 2, 64), gen(2), BF)
    keep = c.k.clone()
    short = cs.Pages(c.k, c.v, c.table[:, :2].contiguous(), c.length)
    cs.cs_paged_append(short, k, k)                                   # rows of stream 1 (positions 40..) have no column
    t0 = c.table[0].cpu()
    for i in range(3):
        assert torch.equal(c.k[int(t0[1]), :, 12 + i], k[i])
        keep[int(t0[1]), :, 12 + i] = k[i]
    assert torch.equal(torch.nan_to_num(c.k.float(), nan=1e30), torch.nan_to_num(keep.float(), nan=1e30))


def test_append_many_streams():
    """More streams than a wave has lanes, some without rows."""
    B = 150
    lens, rows = [(7 * b) % 40 for b in range(B)], [b % 4 for b in range(B)]
    c = Cache(lens, rows, 1, 64, 16, BF, pad=2)
    k = randn((c.R, 1, 64), gen(2), BF)
    cs.cs_paged_append(c.pages, k, -k, row0=c.row0)
    table = c.table.cpu()
    for b in range(B):
        for i in range(rows[b]):
            at = lens[b] + i
            assert torch.equal(c.k[int(table[b][at // 16]), :, at % 16], k[c.ends[b] + i]), (b, i)
            assert torch.equal(c.v[int(table[b][at // 16]), :, at % 16], -k[c.ends[b] + i]), (b, i)
            c.k_tok[b][:, at], c.v_tok[b][:, at] = k[c.ends[b] + i], -k[c.ends[b] + i]
    c.check(4)


# ------------------------------------------------------------------------------------------------------
# together, on streams, in graphs
# ------------------------------------------------------------------------------------------------------

def _layer(c, qkv, H, KVH, gains, f, pos, **call):
    q, k = cs.cs_op_qk_norm_rope(qkv[:, :H], qkv[:, H:H + KVH], pos, f, *gains, **call)
    cs.cs_paged_append(c.pages, k, qkv[:, H + KVH:], row0=c.row0, **call)
    return cs.cs_paged_attention(c.pages, q, row0=c.row0, **call)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_steps_of_a_layer(dtype):
    """Norms, append and attention as a serving loop runs them: a prompt in two chunks, then blocks of copied tokens of which
    some are dropped again, against attention over the plain concatenation."""
    H, KVH, hd, P = 8, 2, 64, 16
    c = Cache([0, 0], [400, 400], KVH, hd, P, dtype)
    c.k.fill_(math.nan), c.v.fill_(math.nan)
    c.length.zero_()
    g, f = gen(11), inv_freq_of(hd)
    gains = (1 + 0.1 * randn((hd,), g, F32), 1 + 0.1 * randn((hd,), g, F32))
    keys = [torch.zeros((0, KVH, hd), dtype=dtype, device=DEV) for _ in range(2)]
    vals = [k.clone() for k in keys]
    for rows, kept in (((70, 3), (70, 3)), ((33, 120), (33, 120)), ((11, 11), (4, 11)), ((1, 11), (1, 1)), ((6, 0), (2, 0)), ((1, 1), (1, 1))):
        lens = [k.shape[0] for k in keys]
        c.lens, c.rows, c.ends = lens, list(rows), [0, rows[0], sum(rows)]
        c.row0.copy_(torch.tensor(c.ends))
        c.length.copy_(torch.tensor(lens))
        qkv = randn((sum(rows), H + 2 * KVH, hd), g, dtype)
        pos = torch.cat([torch.arange(n, n + r, device=DEV, dtype=torch.int32) for n, r in zip(lens, rows)])
        got = _layer(c, qkv, H, KVH, gains, f, pos)
        q, k = cs.cs_op_qk_norm_rope(qkv[:, :H], qkv[:, H:H + KVH], pos, f, *gains)
        c.k_tok = [torch.cat([keys[b], k[c.ends[b]:c.ends[b + 1]]]).transpose(0, 1).contiguous() for b in range(2)]
        c.v_tok = [torch.cat([vals[b], qkv[c.ends[b]:c.ends[b + 1], H + KVH:]]).transpose(0, 1).contiguous() for b in range(2)]
        c.close(got, *c.reference(q, 1 / math.sqrt(hd)), hd)
        for b in range(2):
            n = lens[b] + kept[b]
            keys[b], vals[b] = c.k_tok[b].transpose(0, 1)[:n], c.v_tok[b].transpose(0, 1)[:n]


def test_rotation_of_the_append_is_that_of_the_norm_pass():
    """Keys rotated on the way into the pages and keys rotated before are the same bits."""
    a, b = (Cache([9, 33], [5, 7], 2, 128, 16, BF, seed=4) for _ in range(2))
    kv, f = randn((12, 4, 128), gen(8), BF), inv_freq_of(128)
    pos = torch.cat([torch.arange(9, 14, device=DEV, dtype=torch.int32), torch.arange(33, 40, device=DEV, dtype=torch.int32)])
    cs.cs_paged_append(a.pages, kv[:, :2], kv[:, 2:], row0=a.row0, inv_freq=f)
    _, k = cs.cs_op_qk_norm_rope(kv[:, 2:], kv[:, :2], pos, f)
    cs.cs_paged_append(b.pages, k, kv[:, 2:], row0=b.row0)
    assert torch.equal(torch.nan_to_num(a.k.float(), nan=1e30), torch.nan_to_num(b.k.float(), nan=1e30))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [[1, 1, 1], [11, 3, 0], [200, 1, 1]])
def test_captured_layer_follows_the_lengths(rows, dtype):
    """A captured step replayed while the lengths in device memory grow, between eager steps on another cache."""
    H, KVH, hd, P = 8, 2, 128, 16
    lens = [40, 7, 5000]
    c, e = (Cache(lens, [r + 40 for r in rows], KVH, hd, P, dtype, seed=6) for _ in range(2))
    f = inv_freq_of(hd)
    ends = [0, rows[0], rows[0] + rows[1], sum(rows)]
    for x in (c, e):
        x.row0.copy_(torch.tensor(ends))
    qkv = randn((sum(rows), H + 2 * KVH, hd), gen(12), dtype)
    pos = torch.zeros(sum(rows), dtype=torch.int32, device=DEV)
    step = torch.ones(3, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(c, qkv, H, KVH, (None, None), f, pos)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(c, qkv, H, KVH, (None, None), f, pos)
        c.length.add_(step)
    for i in range(4):
        qkv.copy_(randn(qkv.shape, gen(100 + i), dtype))
        pos.copy_(torch.cat([torch.arange(n + i, n + i + r, device=DEV, dtype=torch.int32) for n, r in zip(lens, rows)]))
        want = _layer(e, qkv, H, KVH, (None, None), f, pos)
        e.length.add_(step)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_two_streams_at_once():
    """Calls on two streams with a workspace each give what they give alone."""
    a = Cache([9000, 20011], [11, 11], 2, 128, 64, BF, seed=1)
    b = Cache([4000, 100], [1, 1], 2, 128, 16, BF, seed=2)
    qa, qb = randn((22, 8, 128), gen(1), BF), randn((2, 8, 128), gen(2), BF)
    wa, wb = cs.cs_paged_attention(a.pages, qa), cs.cs_paged_attention(b.pages, qb)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        got.append((cs.cs_paged_attention(a.pages, qa, stream=s1), cs.cs_paged_attention(b.pages, qb, stream=s2.cuda_stream)))
        got.append((cs.cs_paged_attention(a.pages, qa, stream=0), cs.cs_paged_attention(b.pages, qb, stream=torch.cuda.default_stream())))
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, wa) and torch.equal(y, wb)


def test_workspace_of_the_callers():
    c = Cache([9000, 20011], [11, 11], 2, 128, 64, BF)
    q = randn((22, 8, 128), gen(1), BF)
    want = cs.cs_paged_attention(c.pages, q, max_rows=11, max_len=20022)
    need = cs.cs_paged_attention_workspace(c.pages, 8, 22, max_rows=11, max_len=20022)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    assert torch.equal(cs.cs_paged_attention(c.pages, q, max_rows=11, max_len=20022, workspace=ws[:need] if need else None), want)
    assert bool((ws[need:] == 0xA5).all())
    if need:
        with pytest.raises(cs.CopySpecError):
            cs.cs_paged_attention(c.pages, q, max_rows=11, max_len=20022, workspace=ws[:need - 16])


def test_pool_beyond_two_to_the_32_bytes():
    """Pages whose byte offset needs 33 bits and more."""
    P, KVH, hd, n_pages = 256, 8, 128, 10000                          # 5.2 GB a pool
    k = torch.empty((n_pages, KVH, P, hd), dtype=BF, device=DEV)
    v = torch.empty_like(k)
    names = [0, 9999, 4095, 8191, 8192, 9000]
    g = gen(3)
    kt, vt = randn((KVH, len(names) * P, hd), g, BF), randn((KVH, len(names) * P, hd), g, BF)
    for j, n in enumerate(names):
        k[n], v[n] = kt[:, j * P:(j + 1) * P], vt[:, j * P:(j + 1) * P]
    c = Cache([6 * P - 8], [8], KVH, hd, P, BF)
    c.k, c.v, c.k_tok, c.v_tok = k, v, [kt], [vt]
    c.table = torch.tensor([names], dtype=torch.int32, device=DEV)
    c.pages = cs.Pages(k, v, c.table, c.length)
    c.check(32)
    row = randn((8, KVH, hd), g, BF)
    cs.cs_paged_append(c.pages, row, -row)
    assert torch.equal(k[9000, :, P - 8:].transpose(0, 1), row) and torch.equal(v[9000, :, P - 8:].transpose(0, 1), -row)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_results_repeat_bit_for_bit(dtype):
    """Nothing depends on the order in which workgroups finish."""
    c = Cache([3000, 17, 900], [40, 1, 5], 2, 128, 16, dtype, pad=1)
    q, got = c.check(8)
    for _ in range(5):
        assert torch.equal(cs.cs_paged_attention(c.pages, q, row0=c.row0)[:46], got[:46])


def test_no_rows_and_no_streams():
    c = Cache([20], [1], 2, 64, 16, BF)
    empty = torch.empty((0, 4, 64), dtype=BF, device=DEV)
    assert cs.cs_paged_attention(c.pages, empty).shape == (0, 4, 64)
    cs.cs_paged_append(c.pages, empty[:, :2], empty[:, :2])
    cs.cs_op_qk_norm_rope(empty, None, torch.empty(0, dtype=torch.int32, device=DEV), inv_freq_of(64))
    none = cs.Pages(c.k, c.v, c.table[:0], c.length[:0])
    q = torch.full((2, 4, 64), 3.0, dtype=BF, device=DEV)
    out = q.clone()
    cs.cs_paged_attention(none, q, out=out)
    assert torch.equal(out, q)


@pytest.mark.parametrize("hd,H,KVH", [(128, 8, 2), (64, 7, 1), (256, 4, 2)])
@pytest.mark.parametrize("P,L,rows", [(1024, 683, 336), (2048, 1501, 543), (1024, 1, 1021)])
def test_attention_pool_of_one_page(P, L, rows, hd, H, KVH):
    """A pool that ends with its only page, cut into ranges of which the early tiles have nothing: those begin where a tile's
    tokens end, at no multiple of 16, and what they ask for has to lie in the page all the same."""
    c = Cache([L], [rows], KVH, hd, P, BF, seed=hd, spare=0)
    assert c.k.shape[0] == 1
    q = randn((rows, H, hd), gen(1), BF, 2.0)
    want = c.reference(q, 1 / math.sqrt(hd))
    for call in (dict(max_len=L + rows), dict(row0=c.row0), dict(row0=c.row0, max_rows=rows, max_len=L + rows)):
        c.close(cs.cs_paged_attention(c.pages, q, **call), *want, hd)
    # the same page named by every entry of a longer table, and an entry that names none
    twice = torch.tensor([[-1, int(c.table[0, 0]), 1 << 30]], dtype=torch.int32, device=DEV)
    length = torch.tensor([P + L], dtype=torch.int32, device=DEV)
    c.close(cs.cs_paged_attention(cs.Pages(c.k, c.v, twice, length), q), *want, hd)


# ------------------------------------------------------------------------------------------------------
# the largest numbers of rows and workgroups
# ------------------------------------------------------------------------------------------------------

def test_norm_rope_and_append_of_the_most_rows():
    """2^26 rows: their workgroups of four rows have 2^32 threads."""
    R, hd, P = 1 << 26, 8, 32768
    g, f = gen(3), inv_freq_of(hd)
    x = randn((1, 1, hd), g, F32).expand(R, 1, hd)                        # one row, R times
    pos = torch.arange(R, device=DEV, dtype=torch.int32)
    out = torch.full((R, 1, hd), 9.0, dtype=BF, device=DEV)
    cs.cs_op_qk_norm_rope(x, None, pos, f, out=(out, None))
    some = torch.tensor([0, 1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, R // 2, R - 5, R - 4, R - 1], device=DEV)
    want, bound = ref_norm_rope(x[some], None, pos[some], f, 0.0)
    # (a position of 26 bits: two roundings of 2^-53 in the angle on either side, as for far positions)
    tol = bound * (1 + HALF[BF]) + want.abs() * HALF[BF] + x[some].double().abs().amax() * 8 * R * 2.0 ** -53
    assert bool(((out[some].double() - want).abs() <= tol).all())
    assert not bool((out == 9.0).all(-1).any())
    del out
    k, v = randn((1, 1, hd), g, BF).expand(R, 1, hd), randn((1, 1, hd), g, BF).expand(R, 1, hd)
    pool = torch.zeros((2, 2, 1, P, hd), dtype=BF, device=DEV)
    table = torch.full((1, R // P), -1, dtype=torch.int32, device=DEV)    # only the first and the last page exist
    table[0, 0], table[0, -1] = 1, 0
    cs.cs_paged_append(cs.Pages(pool[0], pool[1], table, torch.zeros(1, dtype=torch.int32, device=DEV)), k, v)
    assert torch.equal(pool[0], k[:1].expand(2, 1, P, hd)) and torch.equal(pool[1], v[:1].expand(2, 1, P, hd))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_of_the_most_workgroups(dtype):
    """65536 streams of 256 KV heads, one token each: 2^24 workgroups of 256 threads.  All streams have the same page."""
    B, H, hd, P, L = 65536, 256, 8, 16, 3
    g = gen(4)
    k, v = randn((1, H, P, hd), g, dtype), randn((1, H, P, hd), g, dtype)
    pages = cs.Pages(k, v, torch.zeros((B, 1), dtype=torch.int32, device=DEV), torch.full((B,), L, dtype=torch.int32, device=DEV))
    q = randn((B, H, hd), g, dtype)
    out = cs.cs_paged_attention(pages, q, max_rows=1, max_len=P)
    c = Cache([L], [1], H, hd, P, dtype)
    x = q.double()                                                        # all of them against the definition
    s = torch.stack([(x * k[0, :, t].double()).sum(-1) for t in range(L + 1)]) / math.sqrt(hd)
    d = torch.stack([(x * k[0, :, t].double()).abs().sum(-1) for t in range(L + 1)]).amax(0) / math.sqrt(hd)
    p = torch.softmax(s, 0)
    want, mag = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(L + 1):
        want += p[t][..., None] * v[0, :, t].double()
        mag += p[t][..., None] * v[0, :, t].double().abs()
    c.close(out, want, mag, d[..., None], hd)


def test_parameters_without_autograd():
    """Gains and rows that are parameters of a model give what plain tensors give, where no gradient is recorded."""
    g = gen(6)
    q, gain = randn((5, 4, 64), g, BF), 1 + 0.1 * randn((64,), g, F32)
    want, _ = cs.cs_op_qk_norm_rope(q, q_gain=gain)
    p, pg = torch.nn.Parameter(q.clone()), torch.nn.Parameter(gain.clone())
    with pytest.raises(RuntimeError):
        cs.cs_op_qk_norm_rope(p, q_gain=pg)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            assert torch.equal(cs.cs_op_qk_norm_rope(p, q_gain=pg)[0], want)
    assert torch.equal(cs.cs_op_qk_norm_rope(p.detach(), q_gain=pg.detach())[0], want)


def test_sizes_that_need_more_than_32_bits_are_refused():
    """The C entries take 32 bits: a larger number is not cut to its low bits (2^32 + 5 would be a window of 5)."""
    c = Cache([40, 3], [2, 2], 2, 64, 16, BF)
    q = randn((4, 4, 64), gen(1), BF)
    one = q[:1, :2]
    many = one.expand((1 << 32) + 1, 2, 64)                               # (a view: one row)
    out = torch.empty_like(q)
    big = (1 << 32) + 5
    for call in (lambda: cs.cs_paged_attention(c.pages, q, window=big, out=out), lambda: cs.cs_paged_attention(c.pages, q, max_rows=big, out=out),
                 lambda: cs.cs_paged_attention(c.pages, many, out=many), lambda: cs.cs_paged_append(c.pages, many, many),
                 lambda: cs.cs_op_qk_norm_rope(many, out=(many, None)), lambda: cs.cs_paged_attention_workspace(c.pages, 4, big),
                 lambda: cs.cs_op_qk_norm_rope(one, one[:, :1].expand(1, big, 64), out=(out[:1, :2], one[:, :1].expand(1, big, 64))),
                 lambda: cs.Pages(c.k[:1].expand(big, *c.k.shape[1:]), c.v[:1].expand(big, *c.v.shape[1:]), c.table, c.length)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    assert torch.equal(cs.cs_paged_attention(c.pages, q, window=(1 << 31) - 1), cs.cs_paged_attention(c.pages, q))


def test_broadcast_inputs_and_strides_that_are_never_taken():
    """One row for all, one KV head's pool for all; single rows and heads of outputs have no stride that counts."""
    c = Cache([40, 3], [2, 2], 1, 64, 16, BF)
    q = randn((1, 4, 64), gen(1), BF)
    wide = cs.Pages(c.k.expand(-1, 2, -1, -1), c.v.expand(-1, 2, -1, -1), c.table, c.length)
    want = cs.cs_paged_attention(c.pages, q.expand(4, 4, 64).contiguous())
    c.close(want, *c.reference(q.expand(4, 4, 64).contiguous(), 0.125), 64)
    assert torch.equal(cs.cs_paged_attention(wide, q.expand(4, 4, 64)), want)
    one = torch.zeros((1, 1, 64), dtype=BF, device=DEV)
    y, _ = cs.cs_op_qk_norm_rope(q[:, :1], q_gain=torch.ones(64, device=DEV), out=(one.as_strided((1, 1, 64), (0, 0, 1)), None))
    assert torch.equal(one, cs.cs_op_qk_norm_rope(q, q_gain=torch.ones(64, device=DEV))[0][:, :1])
    for call in (lambda: cs.cs_paged_attention(c.pages, q.expand(4, 4, 64), out=q.expand(4, 4, 64)),
                 lambda: cs.cs_op_qk_norm_rope(q.expand(4, 4, 64), out=(q.expand(4, 4, 64), None)),
                 lambda: cs.cs_paged_append(wide, want[:, :2], want[:, :2])):
        with pytest.raises(cs.CopySpecError, match="overlap"):
            call()


class Guarded:
    """Tensors inside larger ones that hold a pattern; the surroundings must keep it."""

    def __init__(self):
        self.all = []

    def like(self, shape, dtype, fill=None):
        n = math.prod(shape) * torch.tensor([], dtype=dtype).element_size()
        raw = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device=DEV)
        self.all.append((raw, n))
        t = raw[4096:4096 + n].view(dtype).view(shape)
        if fill is not None:
            t.fill_(fill)
        return t

    def check(self):
        for raw, n in self.all:
            assert bool((raw[:4096] == 0xA5).all()) and bool((raw[4096 + n:] == 0xA5).all()), "written outside the tensor"


def _claimed(offsets, R):
    """Rows that some stream has, by the offsets brought into 0..R."""
    rows = set()
    for a, e in zip(offsets, offsets[1:]):
        rows |= set(range(min(max(a, 0), R), min(max(e, 0), R)))
    return rows


NO_SENSE = {3: ([0, 100, 3, 6], [-50, 2, 2000000000, 6], [6, 4, 2, 0], [0, -1, -2, -3], [2 ** 31 - 1] * 4, [0, 6, 0, 6]),
            73: ([0, 146] * 37, [146 - 2 * b for b in range(74)], [0] * 73 + [146], [(b * 97) % 300 - 50 for b in range(74)])}


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,hint", [(3, 0), (3, 2), (3, 200), (73, 0), (73, 2), (73, 100)])
def test_row_offsets_that_make_no_sense_stay_inside(B, hint, dtype):
    """Offsets outside 0..R or decreasing: nothing around the output, the workspace (of exactly the size asked for) and the pools is
    written, and rows that no stream has are left as they were.  (Which of the others are computed is not said: a row that two streams
    claim, or one more tile than the rows allow, has no right answer.)"""
    lens = [3000, 40, 1000] + [9] * (B - 3)
    c = Cache(lens, [2] * B, 2, 64, 16, dtype)
    R = 2 * B
    guard = Guarded()
    k, v = guard.like(c.k.shape, dtype), guard.like(c.v.shape, dtype)
    q = randn((R, 4, 64), gen(1), dtype)
    for bad in NO_SENSE[B]:
        k.copy_(c.k), v.copy_(c.v)
        pages = cs.Pages(k, v, c.table, c.length)
        row0 = torch.tensor(bad, dtype=torch.int32, device=DEV)
        call = dict(max_rows=hint, max_len=3002 if hint else 0)
        need = cs.cs_paged_attention_workspace(pages, 4, R, row0=True, **call)
        ws, out = guard.like((need,), torch.uint8) if need else None, guard.like((R, 4, 64), dtype, 5.0)
        cs.cs_paged_attention(pages, q, row0=row0, out=out, workspace=ws, **call)
        rows = _claimed(bad, R)
        for r in range(R):
            if r not in rows:
                assert bool((out[r] == 5.0).all()), (bad, r)
        assert torch.equal(torch.nan_to_num(k, nan=1e30), torch.nan_to_num(c.k, nan=1e30))
        # appended rows lie in the slots that the streams' lengths and the offsets name, and nowhere else
        cs.cs_paged_append(pages, q[:, :2], q[:, :2], row0=row0)
        slots = torch.zeros((k.shape[0], 16), dtype=torch.bool)
        table = c.table.cpu()
        for b, (a, e) in enumerate(zip(bad, bad[1:])):
            for i in range(min(max(e, 0), R) - min(max(a, 0), R)):
                at = lens[b] + i
                if at < 16 * table.shape[1] and 0 <= int(table[b][at // 16]) < k.shape[0]:
                    slots[int(table[b][at // 16]), at % 16] = True
        rest = ~slots.to(DEV)
        for new, old in ((k, c.k), (v, c.v)):
            x, y = new.permute(0, 2, 1, 3)[rest], old.permute(0, 2, 1, 3)[rest]
            assert torch.equal(torch.nan_to_num(x, nan=1e30), torch.nan_to_num(y, nan=1e30)), bad
        guard.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("P", [16, 1024])
@pytest.mark.parametrize("rows", [1, 4, 11, 13, 33, 70, 150, 300])
def test_attention_equal_rows_without_offsets(rows, P, dtype):
    """Equal shares, with right hints, none and too small ones, into guarded outputs with guarded workspaces of exactly the size."""
    c = Cache([0, 31, 257, 1100], [rows] * 4, 2, 128, P, dtype, seed=rows)
    q = randn((4 * rows, 8, 128), gen(3), dtype, 2.0)
    want = c.reference(q, 1 / math.sqrt(128))
    guard = Guarded()
    for call in (dict(max_rows=rows, max_len=1100 + rows), {}, dict(max_rows=1, max_len=16)):
        need = cs.cs_paged_attention_workspace(c.pages, 8, 4 * rows, **call)
        ws, out = guard.like((need,), torch.uint8) if need else None, guard.like(q.shape, dtype, 7.0)
        c.close(cs.cs_paged_attention(c.pages, q, out=out, workspace=ws, **call), *want, 128)
    guard.check()
