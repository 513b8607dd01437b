"""Rotary positions on the GPU against the oracle in 64 bits.

Tolerance, value by value: one rounding to the output's type, and the fp32 arithmetic before it.  The angle, in half turns of at most 1, is cut to 32 bits (2^-25
of a half turn, 2^-23.3 radians), sine and cosine are off by 2^-23 at most and stretched (2^-24), two products are added (3 times 2^-24): under 2^-21 of
scale (|a| + |b|)."""
import numpy as np
import pytest

from oracle import cache as C
from test_gpu_residual import HALF, Bench, host, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2012_03837_amd import kernels
    return kernels


def table(rot, base=10000.0, factor=1.0):
    return C.rotary_frequencies(rot, base, factor, 1.0, 32.0, 4096.0)


def check(got, x, pos, freq, rot, interleaved, scale, back, dtype):
    ref = C.rotary(x.astype(np.float64), pos, freq, rot, interleaved, scale, back)
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    more = np.zeros_like(ref)
    more[..., one] = more[..., two] = 2.0 ** -21 * abs(scale) * (np.abs(x[..., one]) + np.abs(x[..., two]))
    assert near(got.reshape(ref.shape), ref, HALF[dtype], more)
    assert np.array_equal(got.reshape(ref.shape)[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("rows,heads,dh,rot,shift", [(1, 1, 2, 2, 0), (1, 24, 64, 64, 0), (5, 9, 80, 32, 0), (3, 2, 64, 40, 0), (130, 3, 33, 12, 1), (2055, 5, 16, 16, 0),
                                                     (700, 7, 24, 24, 0), (40, 3, 512, 512, 0), (1029, 12, 64, 64, 1)])
def test_forward_and_backward(K, dtype, interleaved, rows, heads, dh, rot, shift):
    import torch
    b = Bench(dtype, rows + dh, shift)
    pos = b.rng.integers(-2 ** 20, 2 ** 20, rows).astype(np.int32)
    pos[: 3] = np.array([0, 2 ** 31 - 1, -2 ** 31])[:min(rows, 3)]
    # positions of 2^31 turn the first pair 2^31 radians: 2^-22 of one is what 64 bits leave of the product
    pos[np.abs(pos.astype(np.int64)) > 2 ** 28] //= 8
    freq = table(rot, factor=8.0)
    pd, fd = torch.from_numpy(pos).cuda(), torch.from_numpy(freq).cuda()
    x = b.rnd(rows, heads, dh)
    xd, y = b.dev(x.reshape(rows, -1)), b.room((rows, heads * dh))
    for back in (0, 1):
        K.lpk_rotary(dtype, xd, y, pd, fd, rows, 1, heads, dh, rot, interleaved, 1.25, back)
        check(host(y), x, pos, freq, rot, interleaved, 1.25, back, dtype)
    inplace = b.dev(x.reshape(rows, -1))
    K.lpk_rotary(dtype, inplace, inplace, pd, fd, rows, 1, heads, dh, rot, interleaved, 1.25, 1)
    assert torch.equal(inplace, y) and b.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("wide", [0, 8, 5])
def test_part_of_wider_rows(K, dtype, wide):
    """The q and k columns of qkv, positions by row number: the columns beside them stay."""
    import torch
    b = Bench(dtype, wide)
    B, S, H, dh = 3, 37, 4, 32
    n, ld = 2 * H * dh, 3 * H * dh + wide
    x, freq = b.rnd(B * S, ld), table(dh)
    xd, fd = b.dev(x), torch.from_numpy(freq).cuda()
    K.lpk_rotary(dtype, xd[:, :n], xd[:, :n], None, fd, B * S, S, 2 * H, dh, dh)
    got = host(xd)
    check(got[:, :n], x[:, :n].reshape(B * S, 2 * H, dh), np.tile(np.arange(S), B), freq, dh, 0, 1.0, 0, dtype)
    assert np.array_equal(got[:, n:], x[:, n:]) and b.guards_stand()


def test_frequencies(K):
    for args in ((64, 10000.0, 1.0, 1.0, 1.0, 0.0), (10, 500000.0, 8.0, 1.0, 4.0, 8192.0), (64, 10000.0, 4.0, float("inf"), float("inf"), 0.0), (2, 10.0, 2.0, 3.0, 3.0, 100.0)):
        assert np.allclose(K.lpk_rotary_frequencies(*args).numpy(), C.rotary_frequencies(*args), rtol=1e-14)


def test_infinities_stay_in_their_pair(K):
    import torch
    b = Bench(0, 1)
    x = b.rnd(4, 2, 16)
    x[1, 0, 3], x[2, 1, 15] = np.inf, np.nan
    y = b.room((4, 32))
    K.lpk_rotary(0, b.dev(x.reshape(4, -1)), y, torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda"), torch.from_numpy(table(12)).cuda(), 4, 1, 2, 16, 12)
    bad = ~np.isfinite(host(y).reshape(4, 2, 16))
    want = np.zeros_like(bad)
    want[1, 0, [3, 9]] = want[2, 1, 15] = True
    assert np.array_equal(bad, want)


def test_under_a_replayed_graph_and_on_another_stream(K):
    import torch
    b = Bench(1, 2)
    x, pos, freq = b.dev(b.rnd(65, 128)), torch.arange(65, dtype=torch.int32, device="cuda"), torch.from_numpy(table(64)).cuda()
    y, eager = b.room((65, 128)), b.room((65, 128))
    K.lpk_rotary(1, x, y, pos, freq, 65, 1, 2, 64, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        K.lpk_rotary(1, x, y, pos, freq, 65, 1, 2, 64, 64)
    for i in range(4):
        pos += 1000 * i
        y.zero_()
        graph.replay()
        K.lpk_rotary(1, x, eager, pos, freq, 65, 1, 2, 64, 64)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)


def test_offsets_past_32_bits(K):
    """The last rows of a matrix of 4.3 GB are those of a small one."""
    import torch
    rows, ld = 8, 1 << 28
    big = torch.empty(rows, ld, device="cuda", dtype=torch.bfloat16)
    freq, pos = torch.from_numpy(table(64)).cuda(), torch.arange(rows, dtype=torch.int32, device="cuda")
    small = torch.randn(rows, 128, device="cuda").bfloat16()
    big[:, :128] = small
    want = torch.empty_like(small)
    K.lpk_rotary(1, small, want, pos, freq, rows, 1, 2, 64, 64)
    K.lpk_rotary(1, big[:, :128], big[:, :128], pos, freq, rows, 1, 2, 64, 64)
    assert torch.equal(big[:, :128], want)


def test_in_front_of_attention(K):
    """A layer's attention in training: qkv is turned, attended over, and the gradient comes back through both; against differences of the oracle."""
    import torch
    b = Bench(0, 7)
    B, S, H, dh = 2, 19, 2, 16
    x, do, freq = b.rnd(B * S, 3 * H * dh), b.rnd(B * S, H * dh), table(dh)
    fd = torch.from_numpy(freq).cuda()
    qkv, o, lse, delta, dqkv = b.dev(x), b.room((B * S, H * dh)), b.room((B, H, S)), b.room((B, H, S)), b.room((B * S, 3 * H * dh))
    n = 2 * H * dh
    K.lpk_rotary(0, qkv[:, :n], qkv[:, :n], None, fd, B * S, S, 2 * H, dh, dh)
    K.lpk_attention_fwd(0, qkv, o, lse, B, S, H, dh)
    K.lpk_attention_bwd(0, qkv, o, lse, b.dev(do), dqkv, delta, B, S, H, dh)
    K.lpk_rotary(0, dqkv[:, :n], dqkv[:, :n], None, fd, B * S, S, 2 * H, dh, dh, backward=1)

    def forward(z):
        z = z.copy()
        z[:, :n] = C.rotary(z[:, :n].reshape(B * S, 2 * H, dh), np.tile(np.arange(S), B), freq, dh, False).reshape(B * S, n)
        q, k, v = (z[:, i * H * dh:(i + 1) * H * dh].reshape(B, S, H, dh).transpose(0, 2, 1, 3) for i in range(3))
        s = q @ k.transpose(0, 1, 3, 2) / np.sqrt(dh)
        s = np.where(np.tril(np.ones((S, S), bool)), s, -np.inf)
        w = np.exp(s - s.max(-1, keepdims=True))
        return ((w / w.sum(-1, keepdims=True)) @ v).transpose(0, 2, 1, 3).reshape(B * S, H * dh)

    x64 = x.astype(np.float64)
    assert np.abs(host(o) - forward(x64)).max() < 1e-5
    got = host(dqkv)
    for r, c in [(0, 0), (5, 20), (18, 33), (20, 63), (37, 5), (30, 40), (3, 70)]:
        e = np.zeros_like(x64)
        e[r, c] = 1e-5
        diff = ((forward(x64 + e) - forward(x64 - e)) * do).sum() / 2e-5
        assert abs(got[r, c] - diff) < 2e-5 * max(1.0, abs(diff)), (r, c)
