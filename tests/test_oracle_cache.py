"""The oracle's rotary positions, 8-bit cache and attention over it, pinned by properties and by torch on the CPU."""
import numpy as np
import pytest
import torch

from oracle import cache as C


# ------------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_scores_depend_on_distance(interleaved):
    rng = np.random.default_rng(0)
    freq = C.rotary_frequencies(12, 10000.0, 1.0, 1.0, 1.0, 0.0)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    turn = lambda x, p: C.rotary(x, [p], freq, 12, interleaved)  # noqa: E731
    assert np.isclose((turn(q, 107) * turn(k, 100)).sum(), (turn(q, 7) * turn(k, 0)).sum(), rtol=1e-12)
    assert np.array_equal(turn(k, 0), k) and np.array_equal(turn(k, 5)[..., 12:], k[..., 12:])
    # as a complex number
    y = turn(k, 3)
    a, b = (k[..., 0:12:2], k[..., 1:12:2]) if interleaved else (k[..., :6], k[..., 6:12])
    c, d = (y[..., 0:12:2], y[..., 1:12:2]) if interleaved else (y[..., :6], y[..., 6:12])
    assert np.allclose(c + 1j * d, (a + 1j * b) * np.exp(3j * freq), rtol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_gradient_against_differences(interleaved):
    rng = np.random.default_rng(1)
    freq, pos = C.rotary_frequencies(6, 100.0, 4.0, 1.0, 4.0, 64.0), [3, -17, 100000]
    x, dy = rng.standard_normal((3, 2, 9)), rng.standard_normal((3, 2, 9))
    dx = C.rotary(dy, pos, freq, 6, interleaved, 1.3, backward=True)
    f = lambda z: (C.rotary(z, pos, freq, 6, interleaved, 1.3) * dy).sum()  # noqa: E731
    # the columns behind the rotated part are copied, not stretched
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = 1e-3
        assert abs((f(x + e) - f(x - e)) / 2e-3 - dx[at]) < 1e-9


def test_rotary_frequencies():
    f = C.rotary_frequencies(8, 10000.0, 8.0, 1.0, 32.0, 4096.0)
    plain = 10000.0 ** (-np.arange(4) / 4)
    assert np.allclose(f[:1], plain[:1]) and np.allclose(f[-1:], plain[-1:] / 8)
    assert (f[1:3] < plain[1:3] * 1.0000001).all() and (f[1:3] > plain[1:3] / 8).all()
    assert np.allclose(C.rotary_frequencies(8, 10000.0, 8.0, np.inf, np.inf, 4096.0), plain / 8)


# ------------------------------------------------------------------------------------------------ 8 bits
def test_e4m3_is_torchs():
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.standard_normal(4000) * np.exp2(rng.uniform(-12, 7, 4000)), np.arange(-448, 449) / 2.0, np.arange(64) * 2.0 ** -11])
    x = np.clip(x, -448, 448).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(C.e4m3(x), ref)
    assert (C.e4m3(ref) == ref).all()


def test_scales_are_the_least_powers():
    for most in (448.0, 448.0001, 1.0, 1.75, 1.7500001, 3e38, 1e-45, 2.0 ** -118 * 1.75, 2.0 ** -117):
        s = C.scale_for(most)
        assert np.log2(s) == np.rint(np.log2(s)) and most / s <= 448
        assert s == 2.0 ** -126 or most / (s / 2) > 448
    assert C.scale_for(0.0) == 2.0 ** -126


def _empty(B, L, H, P, dh, pages=None):
    most = -(-L // P)
    pages = pages or B * most + 1
    table = np.random.default_rng(3).permutation(pages)[:B * most].reshape(B, most)
    return table, np.zeros((pages, H, P, dh)), np.zeros((pages, H, dh, P)), np.full((pages, H), np.nan), np.full((pages, H), np.nan)


def test_appended_rows_come_back_within_half_a_step():
    rng = np.random.default_rng(4)
    table, kp, vp, ks, vs = _empty(2, 40, 3, 16, 8)
    x = rng.standard_normal((60, 3, 8)) * np.exp2(rng.integers(-3, 4, (60, 1, 1)))
    seqs = C.sequences([0, 35, 60], [35, 25], 2, 40, 60, 48)
    for pool, scale, values in ((kp, ks, False), (vp, vs, True)):
        C.append(x, pool, scale, values, seqs, table)
        back = C.read(pool, scale, values, seqs, table, 60)
        s = np.zeros((60, 3))
        for b, (first, n, length) in enumerate(seqs):
            for t in range(n):
                s[first + t] = scale[table[b, t // 16]]
        assert (np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s[..., None] * 2.0 ** -10)).all()


def test_growing_scales_round_twice_at_most():
    """One token after another: the page's scale only grows, and what stands there stays within a step of what went in."""
    rng = np.random.default_rng(5)
    table, kp, _, ks, _ = _empty(1, 16, 1, 16, 4)
    x = rng.standard_normal((16, 1, 4)) * np.exp2(np.arange(16))[:, None, None]
    before = 0.0
    for t in range(16):
        C.append(x[t:t + 1], kp, ks, False, [(0, 1, t + 1)], table)
        s = ks[table[0, 0], 0]
        assert s >= before
        before = s
        back = C.read(kp, ks, False, [(0, t + 1, t + 1)], table, t + 1)
        assert (np.abs(back - x[:t + 1]) <= np.abs(x[:t + 1]) * 2.0 ** -4 + s * 2.0 ** -9).all()


def test_attention_is_torchs():
    rng = np.random.default_rng(6)
    table, kp, vp, ks, vs = _empty(2, 30, 2, 16, 8)
    kp[:], vp[:] = C.e4m3(rng.standard_normal(kp.shape) * 50), C.e4m3(rng.standard_normal(vp.shape) * 50)
    ks[:], vs[:] = 2.0 ** rng.integers(-7, -4, ks.shape), 2.0 ** rng.integers(-7, -4, vs.shape)
    seqs = [(0, 3, 30), (3, 7, 7)]
    q = rng.standard_normal((10, 4, 8))
    o, lse, _, _ = C.attention(q, kp, vp, ks, vs, seqs, table, True)
    for b, (first, n, length) in enumerate(seqs):
        k = C.read(kp, ks, False, [(0, 0, 0)] * b + [(0, length, length)], table, length).transpose(1, 0, 2).repeat(2, 0)
        v = C.read(vp, vs, True, [(0, 0, 0)] * b + [(0, length, length)], table, length).transpose(1, 0, 2).repeat(2, 0)
        mask = torch.arange(length)[None] <= torch.arange(length - n, length)[:, None]
        qs = torch.from_numpy(q[first:first + n].transpose(1, 0, 2))
        ref = torch.nn.functional.scaled_dot_product_attention(qs, torch.from_numpy(k), torch.from_numpy(v), attn_mask=mask)
        assert np.allclose(o[first:first + n], ref.numpy().transpose(1, 0, 2), rtol=1e-12, atol=1e-13)
        s = (qs @ torch.from_numpy(k).transpose(1, 2)) / np.sqrt(8)
        assert np.allclose(lse[first:first + n], torch.logsumexp(s.masked_fill(~mask, -np.inf), 2).numpy().T, rtol=1e-12)


def test_rows_that_see_nothing():
    table, kp, vp, ks, vs = _empty(1, 16, 1, 16, 4)
    o, lse, _, _ = C.attention(np.ones((3, 1, 4)), kp, vp, np.ones_like(ks), np.ones_like(vs), [(0, 3, 1)], table, True)
    assert (o == 0).all() and np.isneginf(lse[:2]).all() and lse[2] == 0
    assert C.sequences([0, 5, 4, 9], [3, 3, 99], 3, 4, 8, 50) == [(0, 0, 3), (0, 0, 3), (0, 0, 50)]
