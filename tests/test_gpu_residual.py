"""Dropout and the residual RMS norm on the GPU against the oracle in 64 bits.

Tolerances, value by value: one rounding to the output's type (2^-8 of it in bf16, 2^-24 in fp32) and, beside it, the fp32 arithmetic before it:
a handful of operations for dropout; for the norm a mean of d squares and products, under 2^-24 * (8 + sqrt(d)) of the
largest term, which is taken of the row's largest value."""
import numpy as np
import pytest

from oracle import ops
from oracle import residual as R

pytestmark = pytest.mark.gpu
HALF = {0: 2.0 ** -24, 1: 2.0 ** -8}


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2012_03837_amd import kernels
    return kernels


class Bench:
    """Device buffers between guards that no call may touch."""

    def __init__(self, dtype, seed, shift=0):
        import torch
        self.dtype, self.rng, self.shift, self.whole = dtype, np.random.default_rng(seed), shift, []
        self.tdt = torch.bfloat16 if dtype else torch.float32

    def rnd(self, *shape):
        a = self.rng.standard_normal(shape).astype(np.float32)
        return ops.bf16_round(a).astype(np.float32) if self.dtype else a

    def room(self, shape, dt=None, shift=None):
        import torch
        dt, shift = dt or self.tdt, self.shift if shift is None else shift
        n = int(np.prod(shape))
        raw = torch.full(((n + 128 + shift) * dt.itemsize,), 0xC2, device="cuda", dtype=torch.uint8)
        flat = raw.view(dt)
        self.whole.append((raw, (64 + shift) * dt.itemsize, n * dt.itemsize))
        return flat[64 + shift:64 + shift + n].view(shape)

    def dev(self, a, dt=None):
        import torch
        t = self.room(a.shape, dt)
        t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
        return t

    def guards_stand(self):
        return all(bool((r[:a] == 0xC2).all()) and bool((r[a + n:] == 0xC2).all()) for r, a, n in self.whole)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def generator(seed, step):
    import torch
    wrap = lambda v: v - (1 << 64) if v >= 1 << 63 else v  # noqa: E731
    return torch.tensor([wrap(seed), wrap(step)], dtype=torch.int64, device="cuda")


def near(got, ref, half, more=0.0):
    return bool((np.abs(got - ref) <= 1.01 * half * np.abs(ref) + more).all())


SEED, STEP = 0xFEDCBA9876543210, 0x123456789


# ------------------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 2049, 100003])
def test_dropout_keeps_what_the_generator_says(K, dtype, shift, n):
    b = Bench(dtype, n, shift)
    x, res = b.rnd(n), b.rnd(n)
    xd, rd, y, dx = b.dev(x), b.dev(res), b.room((n,)), b.room((n,))
    rng = generator(SEED, STEP)
    for p in (0.0, 0.1, 0.75, 1.0):
        K.lpk_dropout(dtype, xd, rd, y, p, rng, 5)
        K.lpk_dropout(dtype, xd, None, dx, p, rng, 5)
        ref = R.dropout(x.astype(np.float64), p, SEED, STEP, 5)
        assert ((host(dx) == 0) == (ref == 0)).all()
        assert near(host(dx), ref, HALF[dtype], 2.0 ** -23 * np.abs(ref).max())
        both = ref + res
        assert near(host(y), both, HALF[dtype], 2.0 ** -22 * (np.abs(ref) + np.abs(res)).max())
    assert b.guards_stand()


def test_dropout_in_place_and_elsewhere(K):
    import torch
    b = Bench(1, 1)
    x, res, rng = b.rnd(5000), b.rnd(5000), generator(3, 4)
    xd, rd, y = b.dev(x), b.dev(res), b.room((5000,))
    K.lpk_dropout(1, xd, rd, y, 0.3, rng, 1)
    for out in (xd, rd):
        a, r = b.dev(x), b.dev(res)
        out = a if out is xd else r
        K.lpk_dropout(1, a, r, out, 0.3, rng, 1)
        assert torch.equal(out, y)
    masks = [R.dropout_kept(5000, 0.3, s, t, u) for s, t, u in ((3, 4, 1), (3, 5, 1), (3, 4, 2), (4, 4, 1), (3, 4 + (1 << 32), 1))]
    for i, (s, t, u) in enumerate(((3, 4, 1), (3, 5, 1), (3, 4, 2), (4, 4, 1), (3, 4 + (1 << 32), 1))):
        K.lpk_dropout(1, b.dev(np.ones(5000, np.float32)), None, y, 0.3, generator(s, t), u)
        assert ((host(y) != 0) == masks[i]).all()
        assert i == 0 or (masks[i] != masks[0]).any()


def test_dropout_drops_infinities(K):
    b = Bench(0, 1)
    x = np.full(4096, np.inf, np.float32)
    x[::3] = np.nan
    y = b.room((4096,))
    K.lpk_dropout(0, b.dev(x), None, y, 0.5, generator(1, 1), 0)
    kept = R.dropout_kept(4096, 0.5, 1, 1, 0)
    got = host(y)
    assert (got[~kept] == 0).all() and np.array_equal(got[kept], x[kept].astype(np.float64), equal_nan=True)


def test_dropout_under_a_replayed_graph(K):
    """Every replay reads the step that stands in memory then."""
    import torch
    b = Bench(1, 2)
    x, rng = b.dev(b.rnd(3000)), generator(11, 0)
    y, eager = b.room((3000,)), b.room((3000,))
    K.lpk_dropout(1, x, None, y, 0.4, rng, 9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        K.lpk_dropout(1, x, None, y, 0.4, rng, 9)
    seen = []
    for step in range(4):
        rng[1] = step
        graph.replay()
        torch.cuda.synchronize()
        K.lpk_dropout(1, x, None, eager, 0.4, rng, 9)
        assert torch.equal(eager, y)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1])


def test_dropout_beyond_32_bit_offsets(K):
    import torch
    n = (1 << 31) + 12345
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    K.lpk_dropout(1, x, None, x, 0.25, generator(SEED, STEP), 2)
    groups = -(-n // 8)
    c = np.zeros((200, 4), np.uint64)
    c[:, 0], c[:, 1], c[:, 2], c[:, 3] = np.arange(groups - 200, groups), 2, STEP & 0xFFFFFFFF, STEP >> 32
    words = R.philox(c, (SEED & 0xFFFFFFFF, SEED >> 32))
    kept = (np.stack([words & 0xFFFF, words >> 16], -1).reshape(-1) >= R.dropout_threshold(0.25))[:n - 8 * (groups - 200)]
    assert np.array_equal(host(x[8 * (groups - 200):]) != 0, kept)


# ------------------------------------------------------------------------------------------------ RMS norm
WIDTHS = [1, 5, 8, 64, 65, 72, 128, 200, 256, 512, 513, 520, 1000, 1024, 1032, 2048, 2056, 2047, 4096, 4104, 8192, 8200, 9001, 16384]


def norm_case(K, dtype, rows, d, p, residual, shift=0, seed=0, accumulate=0, scale=1.0):
    import torch
    b = Bench(dtype, seed + d, shift)
    x, res = b.rnd(rows, d) * np.float32(scale), b.rnd(rows, d) if residual else None
    dy, add = b.rnd(rows, d), b.rnd(rows, d) if residual else None
    g = (1 + 0.2 * b.rng.standard_normal(d)).astype(np.float32)
    rng = generator(SEED, STEP) if p else None
    f32 = torch.float32
    gd, xd, dyd = b.dev(g, f32), b.dev(x), b.dev(dy)
    rd = b.dev(res) if residual else None
    store = b.room((rows, d)) if residual or p else None
    y, rstd = b.room((rows, d)), b.room((rows,), f32)
    y8, s8 = b.room((rows, d), torch.float8_e4m3fn), b.room((rows,), f32)
    K.lpk_rmsnorm_fwd(dtype, xd, rd, gd, store, y, y8, s8, rstd, rows, d, 1e-5, p, rng, 6)
    r = R.dropout(x.astype(np.float64), p, SEED, STEP, 6) + (res if residual else 0.0)
    ry, rr = R.rmsnorm_fwd(r, g.astype(np.float64), 1e-5)
    slack = 2.0 ** -24 * (8 + np.sqrt(d))
    if store is not None:
        assert near(host(store), r, HALF[dtype], 2.0 ** -22 * np.abs(r).max())
    else:
        store, r = xd, x.astype(np.float64)
    assert near(host(rstd), rr, 0.0, slack * rr.max())
    assert near(host(y), ry, HALF[dtype], slack * np.abs(ry).max())
    # 8 bits: the scale, and every value within half a step of e4m3 (2^-4 of it, 2^-10 of the smallest normal number's step)
    top = np.abs(ry).max(1)
    assert near(host(s8), np.where(top > 0, top / 448, 1.0), 0.0, 2 * slack * top.max() / 448)
    ref8 = ry / host(s8)[:, None]
    assert (np.abs(host(y8) - ref8) <= 2.0 ** -4 * np.abs(ref8) + 2.0 ** -10 + slack * 448).all()
    # backward, given the sum and the factors as the call left them
    dres, dx, dg = b.room((rows, d)), b.room((rows, d)), b.room((d,), f32)
    dg.fill_(0.5)
    scratch = b.room((K.lpk_rmsnorm_scratch(rows, d),), f32)
    scratch.fill_(float("nan"))
    ad = b.dev(add) if residual else None
    K.lpk_rmsnorm_bwd(dtype, dyd, store, rstd, gd, ad, dres, dx, dg, rows, d, accumulate, scratch, p, rng, 6)
    rdr, rdg = R.rmsnorm_bwd(dy.astype(np.float64), host(store), host(rstd), g.astype(np.float64))
    rdr = rdr + (add if residual else 0.0)
    # dr is a difference of the terms a rstd and xhat mean(a xhat) rstd, which for d = 1 cancel to the share eps has in the mean (of
    # terms of size t each is off by `slack` t whatever remains of them): the largest term of a row counts, not the largest result
    a = np.abs(dy.astype(np.float64) * g) * host(rstd)[:, None]
    xhat = np.abs(host(store) * host(rstd)[:, None])
    terms = np.maximum(a, xhat * (a * xhat).mean(1, keepdims=True)).max(1, keepdims=True) + np.abs(rdr).max()
    assert near(host(dres), rdr, HALF[dtype], 4 * slack * terms)
    rdx = R.dropout(rdr, p, SEED, STEP, 6)
    assert near(host(dx), rdx, HALF[dtype], 4 * slack * terms / (1 - p))
    # a sum of `rows` terms: 2^-24 of the sum of their sizes
    terms = np.abs(dy.astype(np.float64) * host(store) * host(rstd)[:, None]).sum(0)
    assert (np.abs(host(dg) - rdg - 0.5 * accumulate) <= 2.0 ** -24 * (8 + np.sqrt(rows)) * (terms + 1)).all()
    assert b.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_widths(K, dtype, d):
    norm_case(K, dtype, 37, d, 0.25, True)
    norm_case(K, dtype, 3, d, 0.0, False, seed=1, accumulate=1)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d", [(1, 64), (5, 128), (33, 256), (1000, 64), (2600, 768), (4099, 24), (1, 16384), (2000, 449)])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_rows_and_alignment(K, dtype, rows, d, shift):
    norm_case(K, dtype, rows, d, 0.5, True, shift)
    norm_case(K, dtype, rows, d, 0.0, True, shift, seed=2)
    norm_case(K, dtype, rows, d, 0.1, False, shift, seed=3)


def test_norm_parts_of_the_outputs(K):
    """Every output by itself, the same bits as together; in place; nothing where nothing is wanted."""
    import torch
    b = Bench(1, 3)
    rows, d, f32 = 70, 768, torch.float32
    x, res, g, dy = b.dev(b.rnd(rows, d)), b.dev(b.rnd(rows, d)), b.dev(np.ones(d, np.float32), f32), b.dev(b.rnd(rows, d))
    r, y, rstd, y8, s8 = b.room((rows, d)), b.room((rows, d)), b.room((rows,), f32), b.room((rows, d), torch.uint8), b.room((rows,), f32)
    rng = generator(1, 2)
    K.lpk_rmsnorm_fwd(1, x, res, g, r, y, y8, s8, rstd, rows, d, 1e-5, 0.2, rng, 1)
    y1, y81, s81 = b.room((rows, d)), b.room((rows, d), torch.uint8), b.room((rows,), f32)
    K.lpk_rmsnorm_fwd(1, x, res, g, None, y1, None, None, None, rows, d, 1e-5, 0.2, rng, 1)
    K.lpk_rmsnorm_fwd(1, x, res, g, None, None, y81, s81, None, rows, d, 1e-5, 0.2, rng, 1)
    assert torch.equal(y, y1) and torch.equal(y8, y81) and torch.equal(s8, s81)
    keep = res.clone()
    K.lpk_rmsnorm_fwd(1, x, res, g, res, y1, None, None, None, rows, d, 1e-5, 0.2, rng, 1)     # the stream, updated in place
    assert torch.equal(res, r) and torch.equal(y, y1)
    ws = b.room((K.lpk_rmsnorm_scratch(rows, d),), f32)
    dres, dx, dg = b.room((rows, d)), b.room((rows, d)), b.room((d,), f32)
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, keep, dres, dx, dg, rows, d, 0, ws, 0.2, rng, 1)
    a1, a2, a3 = b.room((rows, d)), b.room((rows, d)), b.room((d,), f32)
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, keep, a1, None, None, rows, d, 0, None, 0.2, rng, 1)
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, keep, None, a2, None, rows, d, 0, None, 0.2, rng, 1)
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, keep, None, None, a3, rows, d, 0, ws, 0.2, rng, 1)
    assert torch.equal(a1, dres) and torch.equal(a2, dx) and torch.equal(a3, dg)
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, keep, keep, dy, dg, rows, d, 0, ws, 0.2, rng, 1)       # over its own inputs
    assert torch.equal(keep, dres) and torch.equal(dy, dx) and torch.equal(dg, a3)
    dg.fill_(3.0)
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, None, dres, None, dg, 0, d, 1, ws)
    assert bool((dg == 3).all())
    K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, None, dres, None, dg, 0, d, 0, ws)
    assert bool((dg == 0).all())
    assert b.guards_stand()


@pytest.mark.parametrize("d", [64, 100, 4096])
def test_norm_rows_of_nothing_and_of_infinities(K, d):
    import torch
    b = Bench(0, 4)
    x = b.rnd(6, d)
    x[1] = 0
    x[2, 1], x[3, 2] = np.inf, np.nan
    x[4] = 1e-30
    x[5] = 3e4
    f32 = torch.float32
    y, y8, s8, rstd = b.room((6, d)), b.room((6, d), torch.float8_e4m3fn), b.room((6,), f32), b.room((6,), f32)
    K.lpk_rmsnorm_fwd(0, b.dev(x), None, b.dev(np.ones(d, np.float32)), None, y, y8, s8, rstd, 6, d, 1e-5)
    got, v8 = host(y), host(y8) * host(s8)[:, None]
    ref, _ = R.rmsnorm_fwd(x[[0, 1, 4, 5]].astype(np.float64), np.ones(d), 1e-5)
    assert near(got[[0, 1, 4, 5]], ref, 2.0 ** -22 * (8 + np.sqrt(d)))
    assert not got[1].any() and host(s8)[1] == 1 and not v8[1].any()
    assert np.isnan(got[3]).any() and np.isnan(host(s8)[3]) and not np.isfinite(got[2, 1])
    assert (np.abs(v8[[0, 4, 5]] - ref[[0, 2, 3]]) <= 2.0 ** -3.9 * np.abs(ref[[0, 2, 3]]) + 2.0 ** -9 * host(s8)[[0, 4, 5], None]).all()


def test_norm_beyond_32_bit_offsets(K):
    import torch
    rows, d, f32 = 262400, 8200, torch.float32
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, d, device="cuda", generator=gen, dtype=torch.bfloat16)
    assert x.numel() > 1 << 31
    g, rstd, y, dg = torch.ones(d, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty(d, device="cuda")
    K.lpk_rmsnorm_fwd(1, x, None, g, None, y, None, None, rstd, rows, d, 1e-5)
    r = host(x[-2:])
    ry, rr = R.rmsnorm_fwd(r, np.ones(d), 1e-5)
    assert near(host(y[-2:]), ry, HALF[1], 1e-5)
    ws = torch.empty(K.lpk_rmsnorm_scratch(rows, d), device="cuda")
    dres = torch.empty_like(x)
    K.lpk_rmsnorm_bwd(1, y, x, rstd, g, None, dres, None, dg, rows, d, 0, ws)
    rdr, _ = R.rmsnorm_bwd(host(y[-2:]), r, rr, np.ones(d))
    assert near(host(dres[-2:]), rdr, HALF[1], 1e-5 * rr.max() * np.abs(ry).max())


def test_norm_replays(K):
    import torch
    b = Bench(1, 5)
    rows, d, f32 = 500, 768, torch.float32
    x, res, g, dy = b.dev(b.rnd(rows, d)), b.dev(b.rnd(rows, d)), b.dev(np.ones(d, np.float32), f32), b.dev(b.rnd(rows, d))
    r, y, rstd = b.room((rows, d)), b.room((rows, d)), b.room((rows,), f32)
    dres, dx, dg, ws = b.room((rows, d)), b.room((rows, d)), b.room((d,), f32), b.room((K.lpk_rmsnorm_scratch(rows, d),), f32)
    rng = generator(1, 2)

    def run():
        K.lpk_rmsnorm_fwd(1, x, res, g, r, y, None, None, rstd, rows, d, 1e-5, 0.2, rng, 1)
        K.lpk_rmsnorm_bwd(1, dy, r, rstd, g, res, dres, dx, dg, rows, d, 0, ws, 0.2, rng, 1)
    run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    outs = (r, y, rstd, dres, dx, dg)
    for i in range(3):
        rng[1] = i
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        run()
        assert all(torch.equal(a, t) for a, t in zip(got, outs))


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [0, 1])
def test_attention_branch_of_a_layer(K, dtype):
    """r = stream + drop(branch), y = norm(r), q k v = y Wqkv^T, linear attention, a norm of every head's row, the product back, and its
    dropped sum with r: outputs and all gradients against the same chain in 64 bits with the generator's masks.  The tolerance is that
    of a chain of n stored values, each rounded once (2^-8 in bf16) and passed on through maps whose factors are of order one:
    6 forward and 12 to the end of the backward pass, added as the independent errors that they are, times 2 for the spread of the
    factors: 2 sqrt(12) 2^-8 / sqrt(3) in the 2-norm; fp32 likewise with the operators' own 3e-6."""
    import torch
    b = Bench(dtype, 7)
    B, S, H, dh, p, f32 = 2, 200, 3, 32, 0.2, torch.float32
    d, T = H * dh, 2 * 200
    w = lambda *s: b.rnd(*s) / np.float32(np.sqrt(s[-1]))  # noqa: E731
    wq, wo = (ops.bf16_round(a).astype(np.float32) if dtype else a for a in (w(3 * d, d), w(d, d)))
    x, stream, dout = b.rnd(T, d), b.rnd(T, d), b.rnd(T, d)
    g1, g2 = ((1 + 0.1 * b.rng.standard_normal(n)).astype(np.float32) for n in (d, dh))
    decay = np.array([-0.5, -0.05, -0.005], np.float32)
    lens = np.array([200, 137], np.int32)
    D = {n: b.dev(a) for n, a in dict(x=x, stream=stream, dout=dout, wq=wq, wo=wo).items()}
    G = {n: b.dev(a, f32) for n, a in dict(g1=g1, g2=g2, decay=decay).items()}
    L = torch.from_numpy(lens).cuda()
    rng = generator(21, 2)
    new = lambda *s, dt=None: b.room(s, dt)  # noqa: E731
    r, y, qkv, o, n2, br, out = new(T, d), new(T, d), new(T, 3 * d), new(T, d), new(T, d), new(T, d), new(T, d)
    rs1, rs2 = new(T, dt=f32), new(T * H, dt=f32)
    ws = lambda n: new(max(1, n), dt=f32)  # noqa: E731
    K.lpk_rmsnorm_fwd(dtype, D["x"], D["stream"], G["g1"], r, y, None, None, rs1, T, d, 1e-5, p, rng, 0)
    K.lpk_gemm(dtype, y, d, 1, D["wq"], d, 1, qkv, 3 * d, 0, T, 3 * d, d)
    K.lpk_linear_attention_fwd(dtype, qkv, G["decay"], L, None, o, None, B, S, H, dh, ws(K.lpk_linear_attention_scratch(B, S, H, dh, 0)))
    K.lpk_rmsnorm_fwd(dtype, o, None, G["g2"], None, n2, None, None, rs2, T * H, dh, 1e-5)
    K.lpk_gemm(dtype, n2, d, 1, D["wo"], d, 1, br, d, 0, T, d, d)
    K.lpk_dropout(dtype, br, r, out, p, rng, 1)
    # backward
    dbr, dn2, do, dqkv, dy, dr, dx = new(T, d), new(T, d), new(T, d), new(T, 3 * d), new(T, d), new(T, d), new(T, d)
    dg1, dg2, dwo, dwq = new(d, dt=f32), new(dh, dt=f32), new(d, d, dt=f32), new(3 * d, d, dt=f32)
    K.lpk_dropout(dtype, D["dout"], None, dbr, p, rng, 1)
    K.lpk_gemm(dtype, dbr, d, 1, D["wo"], d, 0, dn2, d, 0, T, d, d)
    K.lpk_gemm(dtype, dbr, d, 0, n2, d, 0, dwo, d, 1, d, d, T)
    K.lpk_rmsnorm_bwd(dtype, dn2, o, rs2, G["g2"], None, do, None, dg2, T * H, dh, 0, ws(K.lpk_rmsnorm_scratch(T * H, dh)))
    K.lpk_linear_attention_bwd(dtype, qkv, G["decay"], L, None, do, None, dqkv, None, B, S, H, dh,
                               ws(K.lpk_linear_attention_scratch(B, S, H, dh, 1)))
    K.lpk_gemm(dtype, dqkv, 3 * d, 1, D["wq"], d, 0, dy, d, 0, T, d, 3 * d)
    K.lpk_gemm(dtype, dqkv, 3 * d, 0, y, d, 0, dwq, d, 1, 3 * d, d, T)
    K.lpk_rmsnorm_bwd(dtype, dy, r, rs1, G["g1"], D["dout"], dr, dx, dg1, T, d, 0, ws(K.lpk_rmsnorm_scratch(T, d)), p, rng, 0)
    # the same in 64 bits
    t64 = lambda a: torch.tensor(a.astype(np.float64), requires_grad=True)  # noqa: E731
    X, ST, WQ, WO, G1, G2 = (t64(a) for a in (x, stream, wq, wo, g1, g2))
    m0, m1 = (torch.from_numpy(R.dropout(np.ones((T, d)), p, 21, 2, site)) for site in (0, 1))
    RR = ST + X * m0
    RR.retain_grad()
    Y = RR * torch.rsqrt((RR * RR).mean(-1, keepdim=True) + 1e-5) * G1
    q, k, v = ((Y @ WQ.T).reshape(B, S, 3, H, dh).permute(2, 0, 3, 1, 4))
    t = torch.arange(S, dtype=torch.float64)
    W = torch.tril(torch.exp(torch.from_numpy(decay.astype(np.float64))[:, None, None] * (t[:, None] - t[None, :]).clamp(min=0))) / dh ** 0.5
    live = (torch.arange(S)[None, :] < torch.from_numpy(lens.astype(np.int64))[:, None])[:, None, :, None]
    O = (((q @ k.transpose(-1, -2)) * W) @ v * live).permute(0, 2, 1, 3).reshape(T * H, dh)
    N2 = (O * torch.rsqrt((O * O).mean(-1, keepdim=True) + 1e-5) * G2).reshape(T, d)
    OUT = RR + (N2 @ WO.T) * m1
    OUT.backward(torch.tensor(dout.astype(np.float64)))
    tol = 2 * np.sqrt(12) * (2.0 ** -8 / np.sqrt(3) if dtype else 3e-6)
    for name, got, want in (("out", out, OUT), ("dx", dx, X.grad), ("dstream", dr, ST.grad), ("dwq", dwq, WQ.grad), ("dwo", dwo, WO.grad),
                            ("dg1", dg1, G1.grad), ("dg2", dg2, G2.grad)):
        a, c = host(got), want.detach().numpy()
        assert np.linalg.norm(a - c) <= tol * np.linalg.norm(c), (name, np.linalg.norm(a - c) / np.linalg.norm(c))
    assert b.guards_stand()


@pytest.mark.parametrize("d", [64, 100, 1024])
def test_norm_gradients_against_differences(K, d):
    """loss = <dy, y> + <add, r> with dropout and residual.  Along a step t e of x, r moves on a line with the direction drop(e), and r / |r| on
    a circle whose angle has the derivatives |e| / c, |e|^2 / c^2 and 2 |e|^3 / c^3 at most, c the line's distance from 0: the third derivative of r / |r| is
    at most 2 + 3 + 1 times (|e| / c)^3, and a central difference is off by t^2 / 6 of that.  y and r are off by 2^-24 (8 + sqrt d) of
    the row's largest value, the gradients by as much."""
    import torch
    rows, eps, p, t = 40, 1e-5, 0.3, 2.0 ** -5
    b = Bench(0, d)
    x, res, dy, add, e = (b.rnd(rows, d) for _ in range(5))
    g = (1 + 0.2 * b.rng.standard_normal(d)).astype(np.float32)
    rng, f32 = generator(SEED, STEP), torch.float32
    dev = {n: b.dev(a) for n, a in dict(x=x, res=res, dy=dy, add=add, g=g).items()}
    r, y, dres, dx = (b.room((rows, d)) for _ in range(4))
    rstd, dg = b.room((rows,)), b.room((d,))
    unit = 2.0 ** -24 * (8 + np.sqrt(d))

    def loss(at, gain):
        K.lpk_rmsnorm_fwd(0, at, dev["res"], gain, r, y, None, None, rstd, rows, d, eps, p, rng, 3)
        yh, rh = host(y), host(r)
        off = unit * ((np.abs(dy).sum(1) * np.abs(yh).max(1)).sum() + (np.abs(add).sum(1) * np.abs(rh).max(1)).sum())
        return (dy.astype(np.float64) * yh).sum() + (add.astype(np.float64) * rh).sum(), off

    base, off0 = loss(dev["x"], dev["g"])
    rh = host(r)
    K.lpk_rmsnorm_bwd(0, dev["dy"], r, rstd, dev["g"], dev["add"], dres, dx, dg, rows, d, 0,
                      torch.empty(K.lpk_rmsnorm_scratch(rows, d), device="cuda", dtype=f32), p, rng, 3)
    dxh, dgh = host(dx), host(dg)
    # x
    high, low = (b.dev((x + s * t * e).astype(np.float32)) for s in (1, -1))
    step = host(high) - host(low)                            # 2 t e, as rounded
    (a, offa), (c, offc) = loss(high, dev["g"]), loss(low, dev["g"])
    along = np.linalg.norm(R.dropout(step, p, SEED, STEP, 3), axis=1) / 2
    clear = np.linalg.norm(rh, axis=1) - along
    assert (clear > 0).all()
    curve = 2 * (np.linalg.norm(g * dy, axis=1) * np.sqrt(d) * (along / clear) ** 3).sum()
    # <dxh, step>: gradients off by `unit` of their row's largest term
    slack = unit * (np.abs(dxh).max(1) * np.abs(step).sum(1)).sum()
    assert abs(a - c - (dxh * step).sum()) <= curve + offa + offc + slack
    # g: the loss is linear in it
    moved = b.dev((2 * g).astype(np.float32))
    (a, offa) = loss(dev["x"], moved)
    assert abs(a - base - (dgh * g).sum()) <= offa + off0 + unit * (np.abs(dy) * np.abs(host(y))).sum()


def test_norm_of_very_many_rows(K):
    """More rows than a launch has threads for along one axis."""
    import torch
    rows = (1 << 26) + 5
    x = torch.arange(rows, device="cuda", dtype=torch.int32).remainder_(97).sub_(48).float()
    g, y = torch.full((1,), 2.0, device="cuda"), torch.full((rows + 64,), 7.0, device="cuda")
    K.lpk_rmsnorm_fwd(0, x, None, g, None, y, None, None, None, rows, 1, 1e-5)
    # five operations in fp32, each off by half a unit
    assert bool((y[:rows].double() - 2 * x.double() / (x.double() ** 2 + 1e-5).sqrt()).abs().max() <= 5 * 2.0 ** -24 * 2)
    assert bool((y[rows:] == 7).all())


def values_beside_middles(scale):
    """Gains whose quotients by `scale` lie at the middles between two 8-bit numbers and one unit beside them, the largest 448 scale."""
    step = [m * 2.0 ** e / 8 for e in range(-6, 9) for m in range(8, 16)]
    step = [v for v in step if v <= 448]
    mid = np.array([(a + b) / 2 for a, b in zip(step, step[1:])])
    at = (mid * float(scale)).astype(np.float32)
    g = np.concatenate([at, np.nextafter(at, np.float32(0)), np.nextafter(at, np.float32(np.inf))])
    return np.concatenate([g, np.resize(g[::-1], 512 - 1 - g.size), [np.float32(448 * float(scale))]]).astype(np.float32)


@pytest.mark.parametrize("odd", [0, 1])
def test_8_bit_values_are_quotients_rounded_once(K, odd):
    """Rows of 1 and -1 without eps: y = g x exactly, and y8 = e4m3(y / s) with the quotient in fp32."""
    import torch
    rng = np.random.default_rng(9)
    told = 0
    for _ in range(20):
        g = values_beside_middles(np.float32(2.0 ** rng.uniform(-3, 3)))[odd:]
        d = g.size
        x = rng.choice(np.array([-1, 1], np.float32), (2, d))
        b = Bench(0, d)
        y, y8, s8 = b.room((2, d)), b.room((2, d), torch.float8_e4m3fn), b.room((2,))
        K.lpk_rmsnorm_fwd(0, b.dev(x), None, b.dev(g), None, y, y8, s8, None, 2, d, 0.0)
        assert np.array_equal(y.cpu().numpy(), g * x)
        scale = np.float32(g.max()) / np.float32(448)
        assert (s8.cpu().numpy() == scale).all()
        e4m3 = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()  # noqa: E731
        want = e4m3(g / scale)
        assert np.array_equal(y8.float().cpu().numpy(), want * x)
        told += int((e4m3(g * (np.float32(1) / scale)) != want).sum())
    assert told > 20                    # values that a product with 1 / s would have moved


def test_8_bit_rows_with_an_infinity(K):
    """A gain of infinity: its column is NaN, the rest of the row, over an infinite scale, zeros."""
    import torch
    b = Bench(0, 3)
    g = np.ones(64, np.float32)
    g[7] = np.inf
    y8, s8 = b.room((1, 64), torch.float8_e4m3fn), b.room((1,))
    K.lpk_rmsnorm_fwd(0, b.dev(np.ones((1, 64), np.float32)), None, b.dev(g), None, None, y8, s8, None, 1, 64, 1e-5)
    got = host(y8)[0]
    assert np.isnan(got[7]) and not np.delete(got, 7).any() and np.isinf(host(s8)[0])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("rows,d", [(70001, 24), (35001, 100), (17001, 200), (8199, 449), (8195, 768), (12300, 1001), (2500, 2047), (2501, 2048), (2500, 4096),
                                    (700, 8191), (600, 8192), (301, 9001), (301, 16384)])
def test_norm_backward_of_several_rows_a_block(K, dtype, shift, rows, d):
    """Two to four rows one after another in a block's turn, the last turn not full: their gain's gradient, the loads ahead, the numbers drawn again."""
    norm_case(K, dtype, rows, d, 0.25, True, shift, seed=4)


def test_norm_gain_gradient_beyond_32_bit_offsets(K):
    import torch
    rows, d = 262400, 8200
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(rows, d, device="cuda", generator=gen, dtype=torch.bfloat16)
    dy = torch.randn(rows, d, device="cuda", generator=gen, dtype=torch.bfloat16)
    rstd = torch.rand(rows, device="cuda", generator=gen) + 0.5
    g, dg = torch.ones(d, device="cuda"), torch.empty(d, device="cuda")
    K.lpk_rmsnorm_bwd(1, dy, x, rstd, g, None, None, None, dg, rows, d, 0, torch.empty(K.lpk_rmsnorm_scratch(rows, d), device="cuda"))
    want, size = (torch.zeros(d, device="cuda", dtype=torch.float64) for _ in range(2))
    for a in range(0, rows, 8192):
        t = dy[a:a + 8192].double() * x[a:a + 8192].double() * rstd[a:a + 8192, None].double()
        want += t.sum(0)
        size += t.abs().sum(0)
    # sums one after another in each of 1024 blocks, then in 64 groups: 2^-24 of the partial sums for each of the steps of a chain, which are independent
    steps = rows / 1024 + 1024 / 64 + 64
    assert bool(((dg - want).abs() <= 2.0 ** -24 * (8 + steps ** 0.5) * size).all())
