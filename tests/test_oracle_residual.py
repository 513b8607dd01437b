"""Pins of the oracle's residual-chain operators: closed forms, finite differences, torch's autograd, published vectors."""
import numpy as np
import pytest

from oracle import residual as R


def _case(seed=0, B=2, H=2, S=9, dh=3):
    rng = np.random.default_rng(seed)
    q, k, v = (rng.standard_normal((B, H, S, dh)) for _ in range(3))
    return rng, q, k, v, np.array([-0.3, -0.01])


def test_linear_attention_is_the_double_sum():
    rng, q, k, v, g = _case()
    s0 = rng.standard_normal((2, 2, 3, 3))
    lens = np.array([9, 4])
    o, s = R.linear_attention_fwd(q, k, v, g, s0, lens)
    for b in range(2):
        for h in range(2):
            n = lens[b]
            for t in range(9):
                want = np.zeros(3)
                if t < n:
                    want = np.exp(g[h] * (t + 1)) * q[b, h, t] @ s0[b, h]
                    for u in range(t + 1):
                        want = want + np.exp(g[h] * (t - u)) * (q[b, h, t] @ k[b, h, u]) * v[b, h, u]
                np.testing.assert_allclose(o[b, h, t], want / np.sqrt(3), rtol=1e-12, atol=1e-13)
            want = np.exp(g[h] * n) * s0[b, h] + sum(np.exp(g[h] * (n - 1 - u)) * np.outer(k[b, h, u], v[b, h, u]) for u in range(n))
            np.testing.assert_allclose(s[b, h], want, rtol=1e-12)


@pytest.mark.parametrize("g", [np.array([-0.3, 0.0]), np.array([-np.inf, -2.0])])
def test_linear_attention_gradients_by_differences(g):
    rng, q, k, v, _ = _case(1)
    s0, do, ds = rng.standard_normal((2, 2, 3, 3)), rng.standard_normal(q.shape), rng.standard_normal((2, 2, 3, 3))
    lens = np.array([9, 5])

    def loss(q, k, v, s0):
        o, s = R.linear_attention_fwd(q, k, v, g, s0, lens)
        return (o * do).sum() + (s * ds).sum()

    grads = R.linear_attention_bwd(q, k, v, g, do, s0, ds, lens)
    at = [q, k, v, s0]
    for i in range(4):
        d = rng.standard_normal(at[i].shape)
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + 1e-6 * d, at[i] - 1e-6 * d
        np.testing.assert_allclose((loss(*up) - loss(*down)) / 2e-6, (grads[i] * d).sum(), rtol=1e-6, atol=1e-7)


def test_philox_published_vectors():
    """The known answers that the method's authors publish with it."""
    for c, k, want in [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                       ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                       ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
                        (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(x) for x in R.philox(np.array([c], np.uint64), k)[0]) == want


def test_dropout_rates_and_limits():
    x = np.ones(80000)
    for p in (0.0, 0.1, 0.5, 0.9, 1.0):
        y = R.dropout(x, p, 12345678901234567, 3, 2)
        kept = (y != 0).mean()
        assert abs(kept - (1 - p)) <= 5 * np.sqrt(max(p * (1 - p), 1e-9) / x.size) + 2.0 ** -17
        if 0 < p < 1:
            np.testing.assert_allclose(y[y != 0], 65536.0 / (65536 - round(p * 65536)))
    a, b = (R.dropout_kept(8000, 0.5, 1, step, site) for step, site in ((0, 0), (0, 1)))
    assert abs((a == b).mean() - 0.5) < 0.05          # another place: another mask


def test_rmsnorm_vs_torch_autograd():
    import torch
    rng = np.random.default_rng(3)
    r, g, dy = rng.standard_normal((7, 11)), rng.standard_normal(11), rng.standard_normal((7, 11))
    tr, tg = torch.tensor(r, requires_grad=True), torch.tensor(g, requires_grad=True)
    ty = torch.nn.functional.rms_norm(tr, (11,), tg, 1e-5)
    ty.backward(torch.tensor(dy))
    y, rstd = R.rmsnorm_fwd(r, g, 1e-5)
    dr, dg = R.rmsnorm_bwd(dy, r, rstd, g)
    for a, b in ((y, ty.detach()), (dr, tr.grad), (dg, tg.grad)):
        np.testing.assert_allclose(a, b.numpy(), rtol=1e-11, atol=1e-12)
