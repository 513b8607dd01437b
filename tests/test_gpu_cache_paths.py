"""Attention over the 8-bit cache where its kernels take ways of their own.  Tolerances are those of test_gpu_cache but where they are
named."""
import numpy as np
import pytest

from oracle import cache as C
from test_gpu_cache import K, Cache, attend, right  # noqa: F401
from test_gpu_residual import HALF, host

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ the largest score of a tile
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,page", [(1, 64), (1, 16), (20, 64), (130, 64), (130, 32)])
@pytest.mark.parametrize("dh", [16, 32, 64, 96, 128, 192, 256])
def test_largest_scores_of_the_last_columns(K, dtype, T, page, dh):  # noqa: F811
    """Every row sees whole tiles only; a tile's largest score is one token's, comes of the head's last column, which the products add last, and is 2^12 times the
    weight of the tile before: a maximum that is taken too early is too small by that."""
    c = Cache(dtype, 17, [T], [512], 1, dh, page)
    c.ks[:], c.kp[:] = 4.0, C.e4m3(c.kp * 2.0 ** -9)
    c.kp[..., dh - 1] = 0.0
    for tile in range(8):
        pos = tile * 64 + (37 * tile + 11) % 64
        c.kp[c.table[0, pos // page], 0, pos % page, dh - 1] = C.e4m3(12 * (tile + 1) * np.log(2) * np.sqrt(dh) / 4)
    c.load()
    q = c.rnd(c.rows, dh)
    q[:, dh - 1] = 1.0
    o, lse, q, _ = attend(K, c, 1, causal=0, q=q)
    right(c, 1, 0, o, lse, q)



# ------------------------------------------------------------------------------------------------ small weights, small values
def near_of_their_own(c, o, q, causal=0):
    """Every column by what stands in it.  One rounding of the output; a weight as in test_gpu_cache (in 24 bits in fp32, 2^-16 in bf16, 2^-12 with many rows) and in bf16 with many
    rows, whose weights end at 2^-32 of a reference that is 2^8 times the row's largest at most, 2^-24 of that for each token: of its |v|, whatever stands in other columns."""
    ref, _, size, mass = C.attention(q.astype(np.float64).reshape(c.rows, c.Hkv, c.dh), c.kp, c.vp, c.ks, c.vs, c.seqs(), c.table, causal)
    n, many, new = int(c.lens[0]), c.T > 32, int(c.starts[1])
    v = np.abs(c.vp * c.vs[..., None, None])[c.table[0]]                     # [pages, heads, dh, page]
    total = v.sum((0, 3)) if many and c.dtype else 0.0
    rel = 2 * (2 * 2.0 ** -24 * (c.dh + 8) * size + 2.0 ** -22) + {(1, True): 2.0 ** -12, (1, False): 2.0 ** -16}.get((c.dtype, many), 2.0 ** -24) + 2 * 2.0 ** -24 * (n / 16 + 64)
    err = np.abs(host(o)[:new].reshape(ref[:new].shape) - ref[:new])
    assert (err <= 1.01 * HALF[c.dtype] * np.abs(ref[:new]) + rel[:new, :, None] * mass[:new] + 2.0 ** -24 * total).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1, 20, 130])
@pytest.mark.parametrize("up", [6, 9, 14, 20, 30, 60, 100])
@pytest.mark.parametrize("page,dh", [(64, 64), (32, 128), (16, 192)])
def test_values_beside_pages_of_large_scales(K, dtype, T, up, page, dh):  # noqa: F811
    """Every third page has large values in one column, zeros in the others: those are the other pages' values all the same."""
    c = Cache(dtype, 19, [T], [512], 1, dh, page)
    large = c.table[0][1::3]
    c.vp[large, :, 1:], c.vs[large] = 0.0, 2.0 ** up
    c.load()
    o, _, q, _ = attend(K, c, 1, causal=0)
    near_of_their_own(c, o, q)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T", [1, 20, 130])
@pytest.mark.parametrize("down", [4, 9, 14])
def test_small_weights_beside_a_large_one(K, dtype, T, down):  # noqa: F811
    """One token has 2^down times the weight of the others and values in one column only."""
    c = Cache(dtype, 23, [T], [2048], 1, 64, 64)
    p, at = c.table[0, 700 // 64], 700 % 64
    c.kp[..., 63], c.ks[:], c.kp[p, 0, at] = 0.0, 2.0 ** -5, 0.0
    c.kp[p, 0, at, 63] = C.e4m3(down * np.log(2) * 8 * 2.0 ** 5 / 8)
    c.vp[p, 0, 1:, at] = 0.0
    c.load()
    q = c.rnd(c.rows, 64)
    q[:, 63] = 8.0
    o, _, q, _ = attend(K, c, 1, causal=0, q=q)
    near_of_their_own(c, o, q)


# ------------------------------------------------------------------------------------------------ tables of all slots
def test_a_table_with_more_rows_than_sequences(K):  # noqa: F811
    """The first rows of a program's table of slots: its other rows, which name the same pages, are not read."""
    import torch
    c = Cache(1, 29, [1, 40], [70, 200], 2, 64, 32)
    o, lse, q, _ = attend(K, c, 2)
    (k, kn), (v, vn) = c.matrix(128), c.matrix(128)
    c.dtable = torch.cat([c.dtable, c.dtable.flip(0), c.dtable.flip(1)])
    o2, lse2, _, _ = attend(K, c, 2, q=q)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    K.lpk_cache_append(1, k, v, *c.paged(), *c.size())
    for x, pool, scale, dpool, values in ((kn, c.kp, c.ks, c.dkp, False), (vn, c.vp, c.vs, c.dvp, True)):
        C.append(x.reshape(c.rows, 2, 64), pool, scale, values, c.seqs(), c.table)
        assert np.array_equal(host(dpool), pool)
    a, b = torch.zeros_like(k).contiguous(), torch.zeros_like(v).contiguous()
    K.lpk_cache_read(1, a, b, *c.paged(), *c.size())
    assert np.array_equal(host(a), C.read(c.kp, c.ks, False, c.seqs(), c.table, c.rows).reshape(c.rows, -1))


# ------------------------------------------------------------------------------------------------ blocks and their work
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("page,length", [(16, 4217), (64, 4217), (256, 2100), (32, 2049)])
def test_long_axes_that_stay_whole(K, dtype, causal, page, length):  # noqa: F811
    """Enough heads and sequences that no axis is divided, and more than 32 and 64 tiles of 64 tokens a block, whose pages are looked up 32 tiles at a time; some are
    missing around those borders."""
    B, heads, used = 8, 64, -(-length // page)
    c = Cache(dtype, page, [35] + [1] * (B - 1), [60] * B, heads, 16, page, most=-(-used // B) + 1)
    c.table = np.full((B, used), -1, np.int32)
    order = c.rng.permutation(c.pages)
    c.table[0], c.table[1:, 0] = order[:used], order[used:used + B - 1]
    for tile in (32, 64):
        at = tile * 64 // page
        c.table[0, at - 1:at], c.table[0, at + 1:at + 2] = -1, -1
    c.lens = np.array([length] + [9] * (B - 1), np.int32)
    c.load()
    assert K.lpk_cache_attention_scratch(B, c.T, heads, heads, 16, page, used) == 0                  # nothing is divided
    o, lse, q, _ = attend(K, c, 1, causal)
    right(c, 1, causal, o, lse, q)
    assert c.guards_stand()


def ragged(rng, B, T, most):
    """New rows and lengths of B sequences: none, one, T and what lies between; some without rows, some without tokens."""
    new = np.minimum(rng.integers(0, T + 1, B), rng.integers(0, T + 1, B))
    new[rng.integers(0, B, B // 5)], new[rng.integers(0, B, B // 8)] = 1, 0
    new[B // 2] = T
    lens = np.maximum(rng.integers(0, most + 1, B), new)
    lens[rng.integers(0, B, 3)] = most
    lens[(new < 2) & (rng.random(B) < 0.1)] = 0
    return [int(n) for n in new], [int(n) for n in lens]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,T,most,Hkv,G,dh,page,divided", [
    (65, 1, 2500, 1, 2, 16, 16, True), (130, 1, 700, 2, 1, 32, 64, True), (130, 4, 700, 2, 3, 16, 32, True), (200, 1, 300, 1, 4, 64, 64, False),
    (70, 150, 500, 1, 1, 16, 16, False), (130, 45, 700, 4, 1, 16, 64, False), (70, 140, 900, 2, 1, 32, 32, True), (129, 20, 650, 1, 3, 16, 16, True)])
def test_many_sequences(K, dtype, B, T, most, Hkv, G, dh, page, divided):  # noqa: F811
    """More sequences than a wave has lanes, ragged, few rows and many, axes whole and divided."""
    new, lens = ragged(np.random.default_rng(B + T), B, T, most)
    c = Cache(dtype, B, new, lens, Hkv, dh, page)
    assert (K.lpk_cache_attention_scratch(B, c.T, Hkv * G, Hkv, dh, page, c.table.shape[1]) > 0) == divided
    o, lse, q, _ = attend(K, c, G)
    right(c, G, 1, o, lse, q)
    assert c.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,chunk,most", [(12, 300, 900), (64, 200, 400), (90, 130, 700)])
def test_single_tokens_beside_a_chunk(K, dtype, B, chunk, most):  # noqa: F811
    """A server's step: one user's chunk of a prompt among others' single tokens."""
    rng = np.random.default_rng(B)
    new, lens = [1] * B, [int(n) for n in rng.integers(1, most + 1, B)]
    new[B // 3], lens[B // 3] = chunk, most
    c = Cache(dtype, B + 1, new, lens, 1, 64, 64)
    o, lse, q, _ = attend(K, c, 2)
    right(c, 2, 1, o, lse, q)
    assert c.guards_stand()


# ------------------------------------------------------------------------------------------------ the ends of the range
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,lens", [(1, 300), (20, 300), (130, 300), (1, 3000), (130, 3000)])
@pytest.mark.parametrize("of_q,of_k", [(71, -71), (-71, 71), (0, 0)])
@pytest.mark.parametrize("of_v", [-68, 68])
def test_ends_of_the_range(K, dtype, T, lens, of_q, of_k, of_v):  # noqa: F811
    """Queries, keys and values as large and as small as the header allows."""
    c = Cache(dtype, 31, [T], [lens], 1, 64, 64)
    c.ks, c.vs = c.ks * 2.0 ** of_k, c.vs * 2.0 ** of_v
    c.vp[c.vp == 0] = 1.0
    c.load()
    o, lse, q, _ = attend(K, c, 1, q=c.rnd(c.rows, 64) * np.float32(2.0 ** of_q))
    right(c, 1, 1, o, lse, q)
    near_of_their_own(c, o, q, 1)
