"""The 8-bit cache of keys and values and attention over it on the GPU against the oracle in 64 bits.

Tolerances.  Codes and scales: none.  A quotient by a power of two is exact, a code is one rounding of it, and what comes back is that code times the
scale, rounded to the output's type (exact in both).
Attention, value by value: one rounding of the output (2^-8 of it in bf16, 2^-24 in fp32) and what comes before it.  A score is a sum of dh exact products in
32 bits and two factors, off by E = 2^-24 (dh + 8) sum |q_i k_i| dh^-1/2 at most, and so is the maximum; exp2 is off by 2^-22 of itself: a weight is off by
2 E + 2^-22 of itself.  What its parts leave out, each the nearest to what the ones before leave: of two
of bf16 2^-16 of it, of three nothing that counts (2^-24); where a call has many rows, of one of f16 2^-12, of two 2^-23, and of weights under 2^-21 of the
largest (times its values' scale) 2^-32 of that (f16 ends at 2^-25, and the largest stands at 2^7 or more): n 2^-32 448 times the largest scale in all.  The weights' and the products' sums are of a few hundred rounded
terms, one behind another: 2^-24 (n / 16 + 64) of sum w |v|, n tokens.  All are relative to sum w |v|, numerator and denominator together twice."""
import numpy as np
import pytest

from oracle import cache as C
from oracle import ops
from test_gpu_residual import HALF, Bench, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2012_03837_amd import kernels
    return kernels


class Cache(Bench):
    """Pools, table and lengths on both sides, some of the pages nobody's."""

    def __init__(self, dtype, seed, new, lens, Hkv, dh, page, shift=0, spare=3, most=None, packed=True):
        super().__init__(dtype, seed, shift)
        rng = self.rng
        self.B, self.Hkv, self.dh, self.page = len(lens), Hkv, dh, page
        self.T = max(1, max(new))
        most = most or max(1, -(-max(lens) // page))
        self.pages = self.B * most + spare
        self.table = rng.permutation(self.pages)[:self.B * most].reshape(self.B, most).astype(np.int32)
        self.lens = np.array(lens, np.int32)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) if packed else None
        self.rows = int(sum(new)) + (5 if packed else 0)                # five rows of no sequence
        self.kp, self.vp = C.e4m3(np.clip(rng.standard_normal((self.pages, Hkv, page, dh)) * 64, -448, 448)), \
            C.e4m3(np.clip(rng.standard_normal((self.pages, Hkv, dh, page)) * 64, -448, 448))
        self.ks, self.vs = 2.0 ** rng.integers(-7, -4, (self.pages, Hkv)), 2.0 ** rng.integers(-7, -4, (self.pages, Hkv))
        self.load()

    def load(self):
        import torch
        f8 = torch.float8_e4m3fn
        self.dkp, self.dvp = self.room(self.kp.shape, f8, 0), self.room(self.vp.shape, f8, 0)
        self.dkp.copy_(torch.from_numpy(self.kp.astype(np.float32)).cuda().to(f8))
        self.dvp.copy_(torch.from_numpy(self.vp.astype(np.float32)).cuda().to(f8))
        self.dks, self.dvs = self.dev(self.ks.astype(np.float32), torch.float32), self.dev(self.vs.astype(np.float32), torch.float32)
        self.dtable, self.dlens = self.dev(self.table, torch.int32), self.dev(self.lens, torch.int32)
        self.dstarts = None if self.starts is None else self.dev(self.starts, torch.int32)

    def paged(self):
        return (self.dstarts, self.dlens, self.dtable, self.dkp, self.dvp, self.dks, self.dvs)

    def seqs(self):
        return C.sequences(self.starts, self.lens, self.B, self.T, self.rows, self.table.shape[1] * self.page)

    def size(self):
        return (self.B, self.T, self.Hkv, self.dh, self.page)

    def matrix(self, cols, wide=0):
        """A matrix whose rows stand in wider ones, and the numbers in it."""
        a = self.rnd(self.rows, cols + wide)
        return self.dev(a)[:, :cols], a[:, :cols]


def same(dev, ref):
    return np.array_equal(host(dev).reshape(ref.shape), ref.astype(np.float32).astype(np.float64), equal_nan=True)


# ------------------------------------------------------------------------------------------------ writing and reading
LAYOUTS = [  # new rows, lengths, heads, dh, page
    ([1], [1], 1, 16, 16), ([1, 1, 1], [1, 16, 17], 2, 64, 16), ([1, 1], [64, 65], 12, 64, 64), ([33, 0, 7], [33, 5, 40], 3, 48, 32),
    ([70, 1, 130], [200, 1, 131], 2, 128, 64), ([5, 300], [259, 300], 1, 256, 256), ([17, 31], [49, 31], 5, 80, 128)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("new,lens,Hkv,dh,page", LAYOUTS)
@pytest.mark.parametrize("wide,shift", [(0, 0), (24, 0), (3, 1)])
def test_append_and_read(K, dtype, new, lens, Hkv, dh, page, wide, shift):
    import torch
    c = Cache(dtype, dh + page, new, lens, Hkv, dh, page, shift)
    (k, kn), (v, vn) = c.matrix(Hkv * dh, wide), c.matrix(Hkv * dh, wide)
    for pool, scale, dpool, dscale, dx, x, values in ((c.kp, c.ks, c.dkp, c.dks, k, kn, False), (c.vp, c.vs, c.dvp, c.dvs, v, vn, True)):
        x *= np.exp2(c.rng.integers(-6, 7, (c.rows, 1))).astype(np.float32)             # scales that grow, and some that do not
        dx.copy_(torch.from_numpy(x))
        C.append(x.reshape(c.rows, Hkv, dh), pool, scale, values, c.seqs(), c.table)
    for _ in range(2):                                                                  # the same rows again: nothing changes
        K.lpk_cache_append(dtype, k, v, *c.paged(), *c.size())
        assert same(c.dks, c.ks) and same(c.dvs, c.vs)
        assert same(c.dkp, c.kp) and same(c.dvp, c.vp)
    outk, outv = c.room((c.rows, Hkv * dh + wide)), c.room((c.rows, Hkv * dh + wide))
    outk.fill_(7.0), outv.fill_(7.0)
    K.lpk_cache_read(dtype, outk[:, :Hkv * dh], outv[:, :Hkv * dh], *c.paged(), *c.size())
    for out, pool, scale, values in ((outk, c.kp, c.ks, False), (outv, c.vp, c.vs, True)):
        ref = C.read(pool, scale, values, c.seqs(), c.table, c.rows).reshape(c.rows, -1)
        ref[sum(new):] = 7.0                                                            # rows of no sequence
        got = host(out)
        assert np.array_equal(got[:, :Hkv * dh], ops.bf16_round(ref) if dtype else ref) and (got[:, Hkv * dh:] == 7.0).all()
    assert c.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
def test_append_token_by_token(K, dtype):
    """What a page holds moves to larger scales as they come, and its first token starts it anew."""
    c = Cache(dtype, 1, [1, 1], [1, 1], 2, 32, 16, most=3, packed=False)
    for t in range(40):
        x = c.rnd(2, 64) * np.float32(2.0 ** ((t * 7) % 12 - 6))
        xd = c.dev(x)
        c.lens[:] = c.dlens[:] = t + 1
        C.append(x.reshape(2, 2, 32), c.kp, c.ks, False, c.seqs(), c.table)
        C.append(x.reshape(2, 2, 32), c.vp, c.vs, True, c.seqs(), c.table)
        K.lpk_cache_append(dtype, xd, xd, *c.paged(), *c.size())
        assert same(c.dks, c.ks) and same(c.dvs, c.vs) and same(c.dkp, c.kp) and same(c.dvp, c.vp), t
    assert c.guards_stand()


@pytest.mark.parametrize("end,scale", [(448.25, 1), (449, 2)])
def test_append_rounds_as_the_type_says(K, end, scale):
    """Ties, the smallest codes, the largest, and numbers below them all, at a scale of 1 and of 2."""
    x = np.concatenate([np.arange(0, end, 0.5), np.arange(64) * 2.0 ** -11, [2.0 ** -10, 3 * 2.0 ** -11, 2.0 ** -30, 1e-40]]).astype(np.float32)
    x = np.resize(np.concatenate([x, -x]), 16 * 128)
    x[0] = 448
    c = Cache(0, 1, [16], [16], 1, 128, 16)
    d = c.dev(np.concatenate([x.reshape(16, 128), np.zeros((5, 128), np.float32)]))
    C.append(x.reshape(16, 1, 128), c.kp, c.ks, False, c.seqs(), c.table)
    C.append(x.reshape(16, 1, 128), c.vp, c.vs, True, c.seqs(), c.table)
    K.lpk_cache_append(0, d, d, *c.paged(), *c.size())
    p = c.table[0, 0]
    assert c.ks[p, 0] == scale and same(c.dks, c.ks) and same(c.dkp, c.kp) and same(c.dvp, c.vp)


@pytest.mark.parametrize("most", [0.0, 1e-45, 2.0 ** -126, 448 * 2.0 ** -126, 449 * 2.0 ** -126, 1.0, 1.75, np.nextafter(np.float32(1.75), np.float32(2)), 3.4e38])
def test_scales_of_extremes(K, most):
    c = Cache(0, 1, [3], [3], 1, 16, 16)
    x = np.zeros((8, 16), np.float32)
    x[:3] = np.float32(most) * np.linspace(-1, 1, 16, dtype=np.float32)
    x[0, 0] = most
    d = c.dev(x)
    C.append(x.reshape(8, 1, 16), c.kp, c.ks, False, c.seqs(), c.table)
    C.append(x.reshape(8, 1, 16), c.vp, c.vs, True, c.seqs(), c.table)
    K.lpk_cache_append(0, d, d, *c.paged(), *c.size())
    assert same(c.dks, c.ks) and same(c.dkp, c.kp) and same(c.dvs, c.vs) and same(c.dvp, c.vp)


@pytest.mark.parametrize("dtype", [0, 1])
def test_infinities_and_nans_stay_with_their_number(K, dtype):
    import torch
    c = Cache(dtype, 3, [20], [45], 2, 32, 32)
    (k, kn), (v, vn) = c.matrix(64), c.matrix(64)
    for d, x in ((k, kn), (v, vn)):
        x[3, 5], x[4, 40], x[10, 0], x[7, :] = np.inf, -np.inf, np.nan, np.nan
        d.copy_(torch.from_numpy(x))
    C.append(kn.reshape(-1, 2, 32), c.kp, c.ks, False, c.seqs(), c.table)
    C.append(vn.reshape(-1, 2, 32), c.vp, c.vs, True, c.seqs(), c.table)
    K.lpk_cache_append(dtype, k, v, *c.paged(), *c.size())
    assert np.isnan(c.kp).sum() == 35 * 1 + 32 and np.isfinite(c.ks).all()
    assert same(c.dks, c.ks) and same(c.dkp, c.kp) and same(c.dvs, c.vs) and same(c.dvp, c.vp)


def test_pages_and_rows_that_are_not_there(K):
    """Page numbers out of range, rows out of order or more than T, lengths beyond the table and before the rows: nothing of them is written."""
    c = Cache(0, 4, [9, 9, 9, 9], [40, 40, 5, 40], 2, 16, 16)
    c.table[0, 2], c.table[1, 2] = -1, c.pages
    c.starts[4] = 60                                                                    # beyond the rows
    c.lens[3] = 1 << 30
    c.load()
    (k, kn), (v, vn) = c.matrix(32), c.matrix(32)
    C.append(kn.reshape(-1, 2, 16), c.kp, c.ks, False, c.seqs(), c.table)
    C.append(vn.reshape(-1, 2, 16), c.vp, c.vs, True, c.seqs(), c.table)
    K.lpk_cache_append(0, k, v, *c.paged(), *c.size())
    assert same(c.dks, c.ks) and same(c.dkp, c.kp) and same(c.dvs, c.vs) and same(c.dvp, c.vp)
    out = c.room((c.rows, 32))
    out.fill_(7.0)
    outv = out.clone()
    K.lpk_cache_read(0, out, outv, *c.paged(), *c.size())
    ref = C.read(c.kp, c.ks, False, c.seqs(), c.table, c.rows).reshape(c.rows, -1)
    ref[27:] = 7.0
    assert np.array_equal(host(out), ref) and (ref[18:22] == 0).all() and (ref[1:9] == 0).all() and c.guards_stand()


# ------------------------------------------------------------------------------------------------ attention
def attend(K, c, G, causal=1, lse=True, wide=0, q=None):
    import torch
    H = c.Hkv * G
    qd, qn = c.matrix(H * c.dh, wide)
    if q is not None:
        qd.copy_(torch.from_numpy(q))
        qn = host(qd)
    o, ls = c.room((c.rows, H * c.dh + wide)), c.room((c.rows, H), torch.float32) if lse else None
    o.fill_(7.0)
    if lse:
        ls.fill_(7.0)
    ws = c.room((max(1, K.lpk_cache_attention_scratch(c.B, c.T, H, c.Hkv, c.dh, c.page, c.table.shape[1])),), torch.float32, 0)
    K.lpk_cache_attention(c.dtype, qd, *c.paged(), o[:, :H * c.dh], ls, c.B, c.T, H, c.Hkv, c.dh, c.page, causal, ws)
    return o, ls, qn, lambda: K.lpk_cache_attention(c.dtype, qd, *c.paged(), o[:, :H * c.dh], ls, c.B, c.T, H, c.Hkv, c.dh, c.page, causal, ws)


def right(c, G, causal, o, lse, q):
    H = c.Hkv * G
    ref, rl, size, mass = C.attention(q.astype(np.float64).reshape(c.rows, H, c.dh), c.kp, c.vp, c.ks, c.vs, c.seqs(), c.table, causal)
    got, gl = host(o)[:, :H * c.dh].reshape(ref.shape), None if lse is None else host(lse)
    rows = np.ones(c.rows, bool)
    for first, n, _ in c.seqs():
        rows[first:first + n] = False
    assert (host(o)[rows] == 7.0).all() and (gl is None or (gl[rows] == 7.0).all())
    got, ref, mass, size, rl = got[~rows], ref[~rows], mass[~rows], size[~rows], rl[~rows]
    E = 2.0 ** -24 * (c.dh + 8) * size
    n = max(c.lens.max(), 1)
    many = c.T * G > 32
    rel = 2 * (2 * E + 2.0 ** -22) + {(1, True): 2.0 ** -12, (0, True): 2.0 ** -23, (1, False): 2.0 ** -16, (0, False): 2.0 ** -24}[c.dtype, many] + 2 * 2.0 ** -24 * (n / 16 + 64)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    err = np.abs(got - ref)[ok] - (1.01 * HALF[c.dtype] * np.abs(ref) + rel[..., None] * mass + (n * 2.0 ** -32 * 448 * np.nanmax(c.vs) if many else 0.0))[ok]
    assert err.size == 0 or err.max() <= 0, err.max()
    if gl is not None:
        gl = gl[~rows]
        assert np.array_equal(np.isneginf(gl), np.isneginf(rl)) and np.array_equal(np.isnan(gl), np.isnan(rl))
        fin = np.isfinite(rl)
        assert (np.abs(gl[fin] - rl[fin]) <= (E + 2.0 ** -22 * (1 + np.abs(rl)) + 2.0 ** -24 * (n / 16 + 64))[fin]).all()


SHAPES = [  # new rows, lengths, heads of the cache, queries a head, dh, page
    ([1], [1], 1, 1, 64, 16), ([1, 1, 1, 1], [63, 64, 65, 0], 2, 1, 64, 64), ([1, 1, 1], [300, 17, 129], 2, 4, 128, 32), ([1, 1], [1000, 31], 3, 3, 80, 16),
    ([1] * 6, [1, 2, 400, 700, 55, 16], 1, 17, 48, 256), ([1, 1], [90, 700], 1, 40, 16, 64), ([3, 0, 2], [100, 60, 2], 2, 2, 64, 16), ([16, 5], [16, 150], 2, 1, 32, 32),
    ([7, 9], [70, 300], 1, 5, 96, 128), ([64, 33], [64, 333], 2, 1, 64, 64), ([70, 200, 1], [70, 201, 90], 1, 2, 64, 32), ([130], [257], 2, 1, 128, 64),
    ([40, 17], [100, 17], 1, 3, 112, 16), ([20, 90], [20, 190], 1, 1, 192, 64), ([33], [120], 2, 2, 256, 32), ([129, 5, 64], [400, 3, 64], 1, 1, 16, 16),
    ([250], [250], 1, 2, 80, 256), ([65, 300], [700, 300], 1, 1, 144, 64), ([8, 4], [90, 300], 1, 4, 64, 64), ([11, 3], [90, 300], 2, 3, 128, 16), ([4], [200], 1, 7, 224, 32)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("new,lens,Hkv,G,dh,page", SHAPES)
def test_attention(K, dtype, causal, new, lens, Hkv, G, dh, page):
    c = Cache(dtype, dh + page + G, new, lens, Hkv, dh, page)
    o, lse, q, _ = attend(K, c, G, causal)
    right(c, G, causal, o, lse, q)
    assert c.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("new,lens,Hkv,G,dh,page,wide,shift", [([1, 1], [90, 200], 2, 2, 64, 64, 8, 0), ([1, 1], [90, 200], 2, 2, 64, 64, 3, 1), ([150], [170], 2, 1, 64, 32, 5, 1),
                                                               ([150], [170], 1, 2, 128, 32, 16, 0)])
def test_attention_of_wider_and_unaligned_rows(K, dtype, new, lens, Hkv, G, dh, page, wide, shift):
    c = Cache(dtype, wide, new, lens, Hkv, dh, page, shift)
    o, lse, q, _ = attend(K, c, G, wide=wide, lse=shift == 0)
    right(c, G, 1, o, lse, q)
    assert (host(o)[:, Hkv * G * dh:] == 7.0).all() and c.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("new,lens,Hkv,G,dh,page", [([1], [5000], 2, 1, 64, 64), ([1] * 5, [4100, 3, 64, 900, 2049], 1, 4, 128, 32), ([1, 1], [3000, 0], 1, 2, 256, 128),
                                                    ([6, 2], [3001, 1500], 2, 2, 64, 16), ([90], [4000], 1, 1, 64, 64), ([100, 30], [2500, 1100], 1, 1, 96, 32)])
def test_attention_over_long_axes(K, dtype, new, lens, Hkv, G, dh, page):
    """Axes that are divided; the pieces join in one order: two runs give the same bits."""
    import torch
    c = Cache(dtype, dh, new, lens, Hkv, dh, page)
    o, lse, q, again = attend(K, c, G)
    right(c, G, 1, o, lse, q)
    one, two = o.clone(), lse.clone()
    again()
    assert torch.equal(o, one) and torch.equal(lse, two) and c.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("new,lens,G,dh", [([1, 1], [200, 330], 1, 64), ([9], [330], 2, 128), ([200], [330], 1, 64), ([140], [2000], 1, 128)])
def test_what_a_row_does_not_see(K, dtype, new, lens, G, dh):
    """NaN in later positions, behind the last token and in unused pages, and large numbers there, do not reach a row; NaN that it sees do."""
    c = Cache(dtype, 5, new, lens, 1, dh, 32)
    for b, n in enumerate(lens):
        last = c.table[b, n // 32] if n % 32 else None
        if last is not None:
            c.kp[last, :, n % 32:], c.vp[last, :, :, n % 32:] = np.nan, np.nan
        for p in c.table[b, -(-n // 32):]:
            c.kp[p], c.vp[p], c.ks[p], c.vs[p] = np.nan, np.nan, np.nan, np.nan
    b, n = 0, lens[0]
    if new[0] > 1:
        at = n - new[0] // 2
        c.vp[c.table[b, at // 32], 0, 3, at % 32] = np.nan                              # a value in one column
        c.kp[c.table[b, (at + 2) // 32], 0, (at + 2) % 32, 1] = np.nan                  # a key: whole rows
    c.load()
    o, lse, q, _ = attend(K, c, G)
    right(c, G, 1, o, lse, q)
    if new[0] > 1:
        bad = np.isnan(host(o)[:sum(new)].reshape(sum(new), G, dh))
        first = new[0] - new[0] // 2
        assert not bad[:first].any() and bad[first, :, 3].all() and bad[first + 2:].all() and bad[first:first + 2].sum() == 2 * G


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("new", [[1, 1, 1], [20, 3, 90]])
def test_pages_that_are_not_there_are_not_seen(K, dtype, new):
    """Pages given back at the front of a sequence, in the middle, all of them."""
    c = Cache(dtype, 6, new, [300, 200, 170], 2, 64, 16)
    c.table[0, :7], c.table[0, 9], c.table[1, :], c.table[2, 5] = -1, c.pages + 5, -7, 1 << 30
    c.load()
    o, lse, q, _ = attend(K, c, 2)
    right(c, 2, 1, o, lse, q)
    assert np.isneginf(host(lse)[new[0]:new[0] + new[1]]).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1, 100])
def test_scores_of_all_sizes(K, dtype, T):
    """Scores up to thousands, one weight takes all; queries of zeros, of infinities and NaN."""
    c = Cache(dtype, 7, [T], [400], 1, 64, 64)
    q = c.rnd(c.rows, 64) * np.float32(100)
    q[0] = 0
    o, lse, q, _ = attend(K, c, 1, q=q)
    right(c, 1, 1, o, lse, q)
    q[0, 3] = np.inf
    if T > 1:
        q[T // 2, 5] = np.nan
    o, lse, q, _ = attend(K, c, 1, q=q)
    got = host(o)[:T]
    assert np.isnan(got[0]).all() and (T == 1 or (np.isnan(got[T // 2]).all() and np.isnan(got).any(1).sum() == 2))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,page", [(1, 64), (1, 16), (130, 64), (130, 32)])
def test_scales_far_apart(K, dtype, T, page):
    """Pages of zeros, whose scales are 2^-126, and of small values between others: their weights count all the same."""
    c = Cache(dtype, 13, [T], [500], 1, 64, page)
    order = c.table[0]
    c.vp[order[::3]], c.vs[order[::3]] = 0.0, 2.0 ** -126
    c.vs[order[1]], c.ks[order[2]] = 2.0 ** -60, 2.0 ** -126
    c.kp[order[2]] = 0.0
    c.load()
    o, lse, q, _ = attend(K, c, 1)
    right(c, 1, 1, o, lse, q)
    c.vp[:], c.vs[:] = 0.0, 2.0 ** -126
    c.load()
    o, lse, q, _ = attend(K, c, 1)
    right(c, 1, 1, o, lse, q)
    assert (host(o)[:T] == 0).all()


@pytest.mark.parametrize("T,lens", [(1, [50, 3000]), (70, [100, 2000])])
def test_attention_under_replayed_graphs(K, T, lens):
    """Two graphs share a workspace; lengths change between replays."""
    import torch
    c = Cache(1, 8, [T, T], lens, 2, 64, 64, packed=False)
    o, lse, q, run = attend(K, c, 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g, stream=s):
            run()
    for i in range(5):
        c.lens[:] = np.maximum(np.array(lens) - 40 * i, T)
        c.dlens.copy_(torch.from_numpy(c.lens))
        o.fill_(7.0)
        graphs[i % 2].replay()
        got = o.clone()
        o.fill_(7.0)
        run()
        torch.cuda.synchronize()
        assert torch.equal(got, o)
    right(c, 2, 1, o, lse, q)


def test_on_another_stream(K):
    import torch
    c = Cache(1, 9, [1, 1], [700, 80], 2, 64, 64)
    o, lse, q, run = attend(K, c, 1)
    want = o.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o.fill_(7.0)
        run()
    s.synchronize()
    assert torch.equal(o, want)


@pytest.mark.parametrize("T", [1, 150])
def test_offsets_past_32_bits(K, T):
    """The last pages of pools of 5 GB answer as the same pages of small ones do, and are written and read alike."""
    import torch
    c = Cache(1, 10, [T, 1], [310, 200], 2, 128, 64)
    o, lse, q, run = attend(K, c, 1)
    (k, _), (v, _) = c.matrix(256), c.matrix(256)
    n = 5 * 2 ** 30 // (2 * 128 * 64)
    big = [torch.empty(n, *p.shape[1:], device="cuda", dtype=p.dtype) for p in (c.dkp, c.dvp, c.dks, c.dvs)]
    for large, small in zip(big, (c.dkp, c.dvp, c.dks, c.dvs)):
        large[n - c.pages:].copy_(small)
    far = (c.dstarts, c.dlens, c.dtable + (n - c.pages), *big)
    o2 = torch.full_like(o, 7.0)
    ws = torch.empty(max(1, K.lpk_cache_attention_scratch(c.B, c.T, 2, 2, 128, 64, c.table.shape[1])), device="cuda")
    K.lpk_cache_attention(1, c.dev(q), *far, o2, None, c.B, c.T, 2, 2, 128, 64, 1, ws)
    assert torch.equal(o, o2)
    K.lpk_cache_append(1, k, v, *c.paged(), *c.size())
    K.lpk_cache_append(1, k, v, *far, *c.size())
    for large, small in zip(big, (c.dkp, c.dvp, c.dks, c.dvs)):
        assert torch.equal(large[n - c.pages:].view(torch.uint8 if small.element_size() == 1 else torch.int32), small.view(torch.uint8 if small.element_size() == 1 else torch.int32))
    a, b = torch.empty_like(k).contiguous(), torch.empty_like(v).contiguous()
    a2, b2 = torch.zeros_like(a), torch.zeros_like(b)
    a.zero_(), b.zero_()
    K.lpk_cache_read(1, a, b, *c.paged(), *c.size())
    K.lpk_cache_read(1, a2, b2, *far, *c.size())
    assert torch.equal(a, a2) and torch.equal(b, b2)


# ------------------------------------------------------------------------------------------------ as a decoder uses them
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("G", [1, 3])
def test_a_prompt_and_then_tokens(K, dtype, G):
    """Prompts of two users, in two chunks, then token by token: positions, cache, attention.  Against attention over the oracle's cache, fed with the rotated
    rows as they were stored, and against the training layout's kernel over what the cache holds."""
    import torch
    Hkv, dh, page, B = 2, 64, 32, 2
    H = Hkv * G
    c = Cache(dtype, 11, [1, 1], [1, 1], Hkv, dh, page, most=4)
    freq = C.rotary_frequencies(dh, 10000.0, 1.0, 1.0, 1.0, 0.0)
    fd = torch.from_numpy(freq).cuda()
    width, total = (H + 2 * Hkv) * dh, np.array([0, 0])
    for new in ([50, 33], [20, 1], [1, 1], [1, 1], [1, 1]):
        c.T, c.rows = max(new), sum(new)
        total = total + new
        c.starts, c.lens = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), total.astype(np.int32)
        c.dstarts, c.dlens = c.dev(c.starts, torch.int32), c.dev(c.lens, torch.int32)
        pos = np.concatenate([np.arange(t - n, t) for t, n in zip(total, new)]).astype(np.int32)
        qkv = c.dev(c.rnd(c.rows, width))
        rot = qkv[:, :(H + Hkv) * dh]
        K.lpk_rotary(dtype, rot, rot, torch.from_numpy(pos).cuda(), fd, c.rows, 1, H + Hkv, dh, dh)
        now = host(qkv)
        q, k, v = qkv[:, :H * dh], qkv[:, H * dh:(H + Hkv) * dh], qkv[:, (H + Hkv) * dh:]
        K.lpk_cache_append(dtype, k, v, *c.paged(), *c.size())
        C.append(now[:, H * dh:(H + Hkv) * dh].reshape(c.rows, Hkv, dh), c.kp, c.ks, False, c.seqs(), c.table)
        C.append(now[:, (H + Hkv) * dh:].reshape(c.rows, Hkv, dh), c.vp, c.vs, True, c.seqs(), c.table)
        assert same(c.dkp, c.kp) and same(c.dvp, c.vp)
        o, lse = c.room((c.rows, H * dh)), c.room((c.rows, H), torch.float32)
        ws = torch.empty(max(1, K.lpk_cache_attention_scratch(B, c.T, H, Hkv, dh, page, 4)), device="cuda")
        K.lpk_cache_attention(dtype, q, *c.paged(), o, lse, B, c.T, H, Hkv, dh, page, 1, ws)
        right(c, G, 1, o, lse, now[:, :H * dh])
    assert c.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
def test_against_the_layer_in_training(K, dtype):
    """A whole sequence through the cache is what lpk_attention_fwd makes of the rows that the cache holds."""
    import torch
    S, H, dh = 130, 2, 64
    c = Cache(dtype, 12, [S], [S], H, dh, 64)
    c.rows = S
    qkv = c.dev(c.rnd(S, 3 * H * dh))
    q, k, v = (qkv[:, i * H * dh:(i + 1) * H * dh] for i in range(3))
    K.lpk_cache_append(dtype, k, v, *c.paged(), *c.size())
    K.lpk_cache_read(dtype, k, v, *c.paged(), *c.size())
    o, lse, ref, rl = c.room((S, H * dh)), c.room((S, H), torch.float32), c.room((S, H * dh)), c.room((1, H, S), torch.float32)
    ws = torch.empty(max(1, K.lpk_cache_attention_scratch(1, S, H, H, dh, 64, c.table.shape[1])), device="cuda")
    K.lpk_cache_attention(dtype, q, *c.paged(), o, lse, 1, S, H, H, dh, 64, 1, ws)
    K.lpk_attention_fwd(dtype, qkv, ref, rl, 1, S, H, dh)
    assert np.abs(host(lse) - host(rl)[0].T).max() < 1e-5
    # lpk_attention_fwd rounds its weights to bf16 in the matrix kernel: half a step of each, and of the output
    assert (np.abs(host(o) - host(ref)) <= (2.0 ** -7 * np.abs(host(ref)) + 2.0 ** -8 * np.abs(host(v)).max() if dtype else 1e-5)).all()
