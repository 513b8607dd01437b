"""Linear attention on the GPU against the oracle's recurrence in 64 bits.

Tolerances (relative 2-norm).  bf16 outputs: one rounding, 2^-8 at most for each value; the operands' parts leave 2^-15 beside it.
fp32 outputs, the states too: every factor and partial sum is off by 2^-24; a chain of c chunks multiplies a decay c times and
adds c times, 64 positions are added inside a chunk, and scores are themselves sums over the head: 2^-24 * (4 + sqrt(64) + sqrt(128) +
c) with c up to 24 here is under 3e-6."""
import numpy as np
import pytest

from oracle import ops
from oracle import residual as R

pytestmark = pytest.mark.gpu
TOL16, TOL32 = 2.0 ** -8 + 2.0 ** -14, 3e-6


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2012_03837_amd import kernels
    return kernels


def relerr(a, ref):
    return float(np.linalg.norm((a - ref).ravel()) / max(np.linalg.norm(ref.ravel()), 1e-30))


class Case:
    """Inputs on the host, buffers on the device between guards that no call may touch."""

    def __init__(self, dtype, B, S, H, dh, seed=0, lens=None, states=True, decay=None, shift=0):
        import torch
        rng = np.random.default_rng(seed)
        self.dtype, self.size = dtype, (B, S, H, dh)
        rnd = lambda *s: (ops.bf16_round(rng.standard_normal(s).astype(np.float32)) if dtype else rng.standard_normal(s)).astype(np.float32)  # noqa: E731
        self.qkv, self.dout = rnd(B * S, 3 * H * dh), rnd(B * S, H * dh)
        self.decay = np.asarray(decay if decay is not None else np.log1p(-np.exp2(-np.linspace(1, 9, H))), np.float32)
        self.lens = None if lens is None else np.asarray(lens, np.int32)
        self.s0 = rng.standard_normal((B, H, dh, dh)).astype(np.float32) if states else None
        self.ds_out = rng.standard_normal((B, H, dh, dh)).astype(np.float32) if states else None
        self.tdt = torch.bfloat16 if dtype else torch.float32
        self.shift, self.whole = shift, []

    def dev(self, a, dt=None):
        import torch
        if a is None:
            return None
        t = self.room(a.shape, dt or (torch.int32 if a.dtype == np.int32 else torch.float32), self.shift if dt is not None else 0)
        t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
        return t

    def room(self, shape, dt, shift=0, value=0.0):
        import torch
        n, pad = int(np.prod(shape)), 64
        flat = torch.full((n + 2 * pad + shift,), -77 if dt == torch.int32 else -77.0, device="cuda", dtype=dt)
        t = flat[pad + shift:pad + shift + n]
        t.fill_(value)
        self.whole.append((flat, pad + shift, n))
        return t.view(*shape)

    def guards_stand(self):
        return all(bool((f[:a] == -77).all()) and bool((f[a + n:] == -77).all()) for f, a, n in self.whole)

    def scratch(self, K, backward):
        import torch
        n = K.lpk_linear_attention_scratch(*self.size, backward)
        return self.room((n,), torch.float32, value=float("nan")) if n else None

    def upload(self):
        self.d = dict(qkv=self.dev(self.qkv, self.tdt), decay=self.dev(self.decay), lens=self.dev(self.lens), s0=self.dev(self.s0),
                      dout=self.dev(self.dout, self.tdt), ds_out=self.dev(self.ds_out))
        return self.d

    def outputs(self):
        import torch
        B, S, H, dh = self.size
        d = self.d
        d["o"], d["dqkv"] = (self.room((B * S, w * H * dh), self.tdt, self.shift, float("nan")) for w in (1, 3))
        d["s_out"], d["ds0"] = (self.room((B, H, dh, dh), torch.float32, value=float("nan")) if self.s0 is not None else None for _ in range(2))
        return d

    def forward(self, K):
        d = self.d
        K.lpk_linear_attention_fwd(self.dtype, d["qkv"], d["decay"], d["lens"], d["s0"], d["o"], d["s_out"], *self.size, self.scratch(K, 0))

    def backward(self, K):
        d = self.d
        K.lpk_linear_attention_bwd(self.dtype, d["qkv"], d["decay"], d["lens"], d["s0"], d["dout"], d["ds_out"], d["dqkv"], d["ds0"],
                                   *self.size, self.scratch(K, 1))

    def heads(self, a):
        B, S, H, dh = self.size
        return np.asarray(a, np.float64).reshape(B, S, H, dh).transpose(0, 2, 1, 3)

    def reference(self):
        B, S, H, dh = self.size
        w = H * dh
        q, k, v = (self.heads(self.qkv[:, i * w:(i + 1) * w]) for i in range(3))
        flat = lambda a: a.transpose(0, 2, 1, 3).reshape(B * S, w)  # noqa: E731
        f64 = lambda a: None if a is None else a.astype(np.float64)  # noqa: E731
        o, s = R.linear_attention_fwd(q, k, v, f64(self.decay), f64(self.s0), self.lens)
        dq, dk, dv, ds = R.linear_attention_bwd(q, k, v, f64(self.decay), self.heads(self.dout), f64(self.s0), f64(self.ds_out), self.lens)
        return dict(o=flat(o), s_out=s, dqkv=np.concatenate([flat(dq), flat(dk), flat(dv)], 1), ds0=ds)

    def check(self, K):
        import torch
        self.upload()
        self.outputs()
        self.forward(K)
        self.backward(K)
        ref = self.reference()
        w = self.size[2] * self.size[3]
        tol = TOL16 if self.dtype else TOL32
        got = {n: None if t is None else t.float().cpu().numpy().astype(np.float64) for n, t in self.d.items() if n in ref}
        assert relerr(got["o"], ref["o"]) <= tol
        for i, n in enumerate("qkv"):
            assert relerr(got["dqkv"][:, i * w:(i + 1) * w], ref["dqkv"][:, i * w:(i + 1) * w]) <= tol, "d" + n
        if self.s0 is not None:
            assert relerr(got["s_out"], ref["s_out"]) <= TOL32
            assert relerr(got["ds0"], ref["ds0"]) <= TOL32
        if self.lens is not None:                      # rows behind a sequence
            B, S = self.size[:2]
            for b in range(B):
                n = int(np.clip(self.lens[b], 0, S))
                assert not got["o"].reshape(B, S, -1)[b, n:].any() and not got["dqkv"].reshape(B, S, -1)[b, n:].any()
        assert self.guards_stand()
        torch.cuda.synchronize()
        return got


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 63, 64, 65, 128, 129, 200])
def test_lengths(K, dtype, S):
    Case(dtype, 2, S, 3, 64, seed=S).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dh", [1, 3, 8, 16, 20, 24, 32, 40, 63, 64, 72, 100, 127, 128])
def test_head_sizes(K, dtype, dh):
    Case(dtype, 2, 150, 2, dh, seed=dh).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,S,H,dh", [(1, 1500, 1, 64), (2, 1031, 3, 32), (1, 769, 2, 128), (3, 512, 2, 16)])
def test_long_axis_in_segments(K, dtype, B, S, H, dh):
    assert K.lpk_linear_attention_scratch(B, S, H, dh, 0) > 0 and K.lpk_linear_attention_scratch(B, S, H, dh, 1) > 0
    Case(dtype, B, S, H, dh, seed=B).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
def test_many_short_sequences_uncut(K, dtype):
    B, S, H, dh = 130, 140, 8, 32
    assert K.lpk_linear_attention_scratch(B, S, H, dh, 0) == K.lpk_linear_attention_scratch(B, S, H, dh, 1) == 0
    Case(dtype, B, S, H, dh).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
def test_very_many_sequences(K, dtype):
    Case(dtype, 9001, 3, 8, 8).check(K)


def test_rows_beyond_32_bit_offsets(K):
    """More than 2^31 elements, one sequence and a state: a decay under which only the last rows count is checked at the end, and the
    state's gradient at the other end.  e^-3 a position: what lies 40 positions back weighs under 1e-52."""
    import torch
    S, H, dh, tail = 720000, 16, 64, 96
    w = H * dh
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn(S, 3 * w, device="cuda", generator=gen, dtype=torch.bfloat16)
    dout = torch.randn(S, w, device="cuda", generator=gen, dtype=torch.bfloat16)
    assert qkv.numel() > 1 << 31
    decay = torch.full((H,), -3.0, device="cuda")
    o, dqkv = torch.empty_like(dout), torch.empty_like(qkv)
    s_out, ds0 = (torch.empty(1, H, dh, dh, device="cuda") for _ in range(2))
    ws = torch.empty(max(K.lpk_linear_attention_scratch(1, S, H, dh, b) for b in (0, 1)), device="cuda")
    K.lpk_linear_attention_fwd(1, qkv, decay, None, None, o, s_out, 1, S, H, dh, ws)
    K.lpk_linear_attention_bwd(1, qkv, decay, None, None, dout, None, dqkv, ds0, 1, S, H, dh, ws)

    def part(t, a, n, i=0):
        return t[a:a + n, i * w:(i + 1) * w].float().cpu().numpy().astype(np.float64).reshape(1, n, H, dh).transpose(0, 2, 1, 3)
    g = np.full(H, -3.0)
    for a, rows in ((S - tail, slice(48, tail)), (0, slice(0, 48)), (S // 2, slice(48, 64))):
        q, k, v, do = (part(t, a, tail, i) for t, i in ((qkv, 0), (qkv, 1), (qkv, 2), (dout, 0)))
        ref_o, ref_s = R.linear_attention_fwd(q, k, v, g)
        grads = R.linear_attention_bwd(q, k, v, g, do)
        assert relerr(part(o, a, tail)[:, :, rows], ref_o[:, :, rows]) <= TOL16, a
        for i in range(3):
            assert relerr(part(dqkv, a, tail, i)[:, :, rows], grads[i][:, :, rows]) <= TOL16, (a, i)
        if a == S - tail:
            assert relerr(s_out.cpu().numpy().astype(np.float64), ref_s) <= TOL32
        if a == 0:
            assert relerr(ds0.cpu().numpy().astype(np.float64), grads[3]) <= TOL32


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("S,dh,lens", [(100, 64, [0, 1, 100, 64]), (700, 64, [0, 700, 129, 65]), (700, 32, [256, 257, -5, 9999]),
                                       (300, 128, [1, 192, 0, 299])])
def test_ragged_batches(K, dtype, S, dh, lens):
    case = Case(dtype, 4, S, 2, dh, seed=S, lens=lens)
    # what stands behind a sequence is not looked at
    for a, w in ((case.qkv, 6 * dh), (case.dout, 2 * dh)):
        x = a.reshape(4, S, w)
        for b, n in enumerate(np.clip(lens, 0, S)):
            x[b, n:] = np.nan
    reference = Case.reference

    def clean(self):
        kept = self.qkv, self.dout
        self.qkv, self.dout = (np.nan_to_num(a) for a in kept)
        out = reference(self)
        self.qkv, self.dout = kept
        return out
    case.reference = clean.__get__(case)
    case.check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("decay", [[0.0, 0.0], [-np.inf, -50.0], [-1e-4, -4.0]])
def test_decays_at_their_limits(K, dtype, decay):
    Case(dtype, 2, 333, 2, 64, seed=5, decay=decay).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("states", [False, True])
def test_unaligned_buffers(K, dtype, states):
    Case(dtype, 2, 300, 2, 64, seed=6, states=states, shift=1).check(K)


def test_states_alone(K):
    """A sequence without positions hands its state through; without states nothing is read or written for them."""
    import torch
    case = Case(1, 2, 0, 2, 64)
    d = case.upload()
    s_out = case.room((2, 2, 64, 64), torch.float32)
    K.lpk_linear_attention_fwd(1, None or d["s0"], d["decay"], None, d["s0"], d["s0"], s_out, 2, 0, 2, 64)
    assert torch.equal(s_out, d["s0"])
    ds0 = case.room((2, 2, 64, 64), torch.float32)
    K.lpk_linear_attention_bwd(1, d["s0"], d["decay"], None, d["s0"], d["s0"], d["ds_out"], d["s0"], ds0, 2, 0, 2, 64)
    assert torch.allclose(ds0, d["ds_out"], rtol=3 * 2.0 ** -24, atol=0)
    assert case.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,S,dh", [(2, 100, 64), (1, 1000, 64), (1, 300, 128)])
def test_state_in_place(K, dtype, B, S, dh):
    import torch
    case = Case(dtype, B, S, 2, dh, seed=3)
    d = case.upload()
    case.outputs()
    case.forward(K)
    o, s = d["o"].clone(), d["s_out"].clone()
    K.lpk_linear_attention_fwd(dtype, d["qkv"], d["decay"], None, d["s0"], d["o"], d["s0"], *case.size, case.scratch(K, 0))
    assert torch.equal(d["o"], o) and torch.equal(d["s0"], s)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,H,dh", [(1, 1, 1), (3, 5, 7), (1, 12, 64), (5, 3, 40), (2, 2, 128), (300, 8, 16), (4, 3, 66)])
def test_step_is_a_call_of_one_position(K, dtype, B, H, dh):
    case = Case(dtype, B, 1, H, dh, seed=dh)
    d = case.upload()
    case.outputs()
    K.lpk_linear_attention_step(dtype, d["qkv"], d["decay"], d["s0"], d["o"], B, H, dh)
    ref = case.reference()
    assert relerr(d["o"].float().cpu().numpy().astype(np.float64), ref["o"]) <= (TOL16 if dtype else TOL32)
    assert relerr(d["s0"].cpu().numpy().astype(np.float64), ref["s_out"]) <= TOL32
    assert case.guards_stand()


def test_step_on_an_unaligned_state(K):
    import torch
    case = Case(1, 3, 1, 2, 64)
    d = case.upload()
    case.outputs()
    state = case.room((3, 2, 64, 64), torch.float32, shift=1)
    state.copy_(d["s0"])
    K.lpk_linear_attention_step(1, d["qkv"], d["decay"], state, d["o"], 3, 2, 64)
    assert relerr(state.cpu().numpy().astype(np.float64), case.reference()["s_out"]) <= TOL32
    assert case.guards_stand()


@pytest.mark.parametrize("dtype", [0, 1])
def test_prompt_then_tokens(K, dtype):
    """A prompt in one call and the rest one by one give what one call gives."""
    B, S, H, dh, cut = 2, 150, 3, 64, 131
    case = Case(dtype, B, S, H, dh, seed=8)
    d = case.upload()
    ref = case.reference()
    rows = d["qkv"].view(B, S, -1)
    state = case.room(d["s0"].shape, d["s0"].dtype)
    o = case.room((B, cut, H * dh), case.tdt)
    prompt = rows[:, :cut].contiguous()
    K.lpk_linear_attention_fwd(dtype, prompt, d["decay"], None, d["s0"], o, state, B, cut, H, dh, case.scratch(K, 0))
    got = [o]
    for t in range(cut, S):
        one = case.room((B, 1, H * dh), case.tdt)
        K.lpk_linear_attention_step(dtype, rows[:, t].contiguous(), d["decay"], state, one, B, H, dh)
        got.append(one)
    import torch
    assert relerr(torch.cat(got, 1).float().cpu().numpy().astype(np.float64).reshape(B * S, -1), ref["o"]) <= (TOL16 if dtype else TOL32)
    assert relerr(state.cpu().numpy().astype(np.float64), ref["s_out"]) <= TOL32


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("S,dh", [(130, 64), (130, 32), (600, 64), (130, 128)])
@pytest.mark.parametrize("which,value", [(0, np.nan), (1, np.inf), (2, np.inf), (2, np.nan), (3, -np.inf), (3, np.nan)])
def test_infinities_reach_no_position_they_must_not(K, dtype, S, dh, which, value):
    """q, k, v or dout with one bad row: forward outputs before it, and gradients that do not depend on it, are those of the clean run."""
    at, H = 77, 2
    runs = []
    for bad in (False, True):
        case = Case(dtype, 1, S, H, dh, seed=4)
        if bad:
            (case.dout if which == 3 else case.qkv)[at, (0 if which == 3 else which * H * dh) + 5] = value       # head 0
        d = case.upload()
        case.outputs()
        case.forward(K)
        case.backward(K)
        runs.append({n: d[n].float().cpu().numpy() for n in ("o", "dqkv")})
    clean, got = runs
    w = H * dh
    cols = {"o": clean["o"], **{n: clean["dqkv"][:, i * w:(i + 1) * w] for i, n in enumerate(("dq", "dk", "dv"))}}
    outs = {"o": got["o"], **{n: got["dqkv"][:, i * w:(i + 1) * w] for i, n in enumerate(("dq", "dk", "dv"))}}
    # positions of head 0 that depend on the row
    after, until, only, none = range(at, S), range(0, at + 1), [at], []
    touched = [dict(o=only, dq=none, dk=until, dv=until), dict(o=after, dq=after, dk=none, dv=until),
               dict(o=after, dq=after, dk=until, dv=none), dict(o=none, dq=only, dk=until, dv=until)][which]
    # a step of the tile products may be taken in another order where a chunk holds such a value: one rounding more
    tol = 2.0 ** -7 if dtype else 1e-5
    for n in outs:
        rows = np.ones(S, bool)
        rows[list(touched[n])] = False
        if rows.any():
            assert np.isfinite(outs[n][rows]).all(), n
            assert relerr(outs[n][rows].astype(np.float64), cols[n][rows].astype(np.float64)) <= tol, n
        assert relerr(outs[n][:, dh:].astype(np.float64), cols[n][:, dh:].astype(np.float64)) <= tol, n        # the other head
    assert not np.isfinite(outs["dv" if which in (0, 1, 3) else "dk"][at, :dh]).all()


@pytest.mark.parametrize("B,S,H,dh", [(2, 300, 2, 64), (1, 1200, 2, 64)])
def test_runs_are_identical_bit_for_bit_and_replay(K, B, S, H, dh):
    """Two eager runs, and a captured pair of calls that is replayed with other inputs between eager work."""
    import torch
    case = Case(1, B, S, H, dh, seed=9)
    d = case.upload()
    case.outputs()
    ws = [case.scratch(K, 0), case.scratch(K, 1)]

    def run():
        K.lpk_linear_attention_fwd(1, d["qkv"], d["decay"], None, d["s0"], d["o"], d["s_out"], *case.size, ws[0])
        K.lpk_linear_attention_bwd(1, d["qkv"], d["decay"], None, d["s0"], d["dout"], d["ds_out"], d["dqkv"], d["ds0"], *case.size, ws[1])
    names = ("o", "s_out", "dqkv", "ds0")
    run()
    first = {n: d[n].clone() for n in names}
    run()
    assert all(torch.equal(first[n], d[n]) for n in names)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    clean = d["qkv"].clone()
    for i in range(3):
        d["qkv"].copy_(clean * (1.0 + 0.5 * i))
        for n in names:
            d[n].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = {n: d[n].clone() for n in names}
        run()
        assert all(torch.equal(got[n], d[n]) for n in names), i


def test_two_streams_at_once(K):
    import torch
    cases = [Case(1, 1, 900, 2, 64, seed=i) for i in range(2)]
    for c in cases:
        c.upload()
        c.outputs()
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(cases, (torch.cuda.Stream(), torch.cuda.Stream())):
            with torch.cuda.stream(s):
                c.forward(K)
                c.backward(K)
    torch.cuda.synchronize()
    for c in cases:
        ref = c.reference()
        for n in ("o", "dqkv"):
            assert relerr(c.d[n].float().cpu().numpy().astype(np.float64), ref[n]) <= TOL16


@pytest.mark.parametrize("S,dh,lens", [(70, 64, [70, 33]), (600, 32, None), (100, 128, None)])
def test_gradients_against_differences(K, S, dh, lens):
    """loss = <dout, o> + <ds_out, s_out> is linear in each of q, k, v and s0: its change over a whole step along one of them is the
    gradient's product with the step, but for the 3e-6 by which outputs and gradients are off."""
    import torch
    c = Case(0, 2, S, 2, dh, seed=S, lens=lens)
    c.upload()
    d = c.outputs()
    w = 2 * dh

    def loss():
        c.forward(K)
        o, s = (d[n].double().cpu().numpy().ravel() for n in ("o", "s_out"))
        a, b = c.dout.astype(np.float64).ravel(), c.ds_out.astype(np.float64).ravel()
        return a @ o + b @ s, 3e-6 * (np.linalg.norm(a) * np.linalg.norm(o) + np.linalg.norm(b) * np.linalg.norm(s))

    c.backward(K)
    grads = {i: d["dqkv"][:, i * w:(i + 1) * w].double().cpu().numpy() for i in range(3)} | {3: d["ds0"].double().cpu().numpy()}
    rng = np.random.default_rng(dh)
    base, off = loss()
    for i in range(4):
        at = d["s0"] if i == 3 else d["qkv"][:, i * w:(i + 1) * w]
        was = at.clone()
        at.add_(torch.from_numpy(rng.standard_normal(tuple(at.shape)).astype(np.float32)).cuda())
        step = (at.double() - was.double()).cpu().numpy()
        moved, off2 = loss()
        at.copy_(was)
        expect = float((grads[i] * step).sum())
        assert abs(moved - base - expect) <= off + off2 + 3e-6 * np.linalg.norm(grads[i]) * np.linalg.norm(step), "qkvs"[i]
        assert abs(expect) > 10 * (off + off2)              # the step is no smaller than what it is measured with


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,S,dh,lens", [(2, 300, 64, None), (1, 1200, 64, None), (2, 900, 64, [900, 411]), (1, 900, 32, None), (1, 900, 128, None), (2, 200, 96, None)])
def test_outputs_do_not_depend_on_what_else_is_asked_for(K, dtype, B, S, dh, lens):
    """o and dqkv are the same bits with and without s_out and ds0."""
    import torch
    case = Case(dtype, B, S, 2, dh, seed=11, lens=lens)
    d = case.upload()
    case.outputs()
    case.forward(K)
    case.backward(K)
    both = d["o"].clone(), d["dqkv"].clone()
    d["s_out"] = d["ds0"] = None
    case.forward(K)
    case.backward(K)
    assert torch.equal(d["o"], both[0]) and torch.equal(d["dqkv"], both[1])


def bf16_call(K, q, k, v, g, s0=None):
    """One sequence and head of 64: o."""
    import torch
    qkv = torch.cat([torch.as_tensor(a, dtype=torch.float32) for a in (q, k, v)], 1).to("cuda", torch.bfloat16)
    S = qkv.shape[0]
    o = torch.empty(S, 64, device="cuda", dtype=torch.bfloat16)
    n = K.lpk_linear_attention_scratch(1, S, 1, 64, 0)
    K.lpk_linear_attention_fwd(1, qkv, torch.tensor([g], device="cuda"), None, None if s0 is None else torch.as_tensor(s0, dtype=torch.float32).cuda(), o, None,
                               1, S, 1, 64, torch.empty(n, device="cuda") if n else None)
    return o.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("which", ["state", "score"])
def test_bf16_operands_keep_32_bits_between_products(K, which):
    """1 + 2^-8 + 2^-20 lies 2^-20 above the middle between two bf16 numbers and becomes the upper one; with 17 bits alone it is the middle, which goes to
    the lower.  As an element of the state, and as a score (whose sum is exact in fp32)."""
    x = 1 + 2.0 ** -8 + 2.0 ** -20
    q, k, v = np.zeros((1, 64)), np.zeros((1, 64)), np.zeros((1, 64))
    if which == "state":
        s0 = np.zeros((1, 1, 64, 64))
        s0[..., 3, :] = 8 * x
        q[0, 3] = 1
        o = bf16_call(K, q, k, v, 0.0, s0)
    else:
        q[0, :3] = 1, 2.0 ** -8, 2.0 ** -20
        k[0, :3] = 1
        v[:] = 8
        o = bf16_call(K, q, k, v, 0.0)
    assert (o == 1 + 2.0 ** -7).all()


def test_bf16_values_keep_32_bits_under_their_decay(K):
    """One key and value, then queries: o_t = l^t v / 8, one product and roundings of 2^-24: of the decay's exponent (up to 4 l^t's) and power, the weight, the value
    times it, the scale, and two for each chunk between; an output is within half a step of its own 8 bits and those."""
    S, g = 200, -0.013
    rng = np.random.default_rng(12)
    q, k, v = np.zeros((S, 64)), np.zeros((S, 64)), np.zeros((S, 64))
    q[:, 5] = k[0, 5] = 1
    v[0] = ops.bf16_round(rng.standard_normal(64).astype(np.float32))
    worst = 0.0
    for i in range(16):
        gi = float(np.float32(g * (1 + i / 16)))
        o = bf16_call(K, q, k, v, gi)
        t = np.arange(S)[:, None]
        exact = np.exp(gi * t) * v[0] / 8
        half = np.exp2(np.floor(np.log2(np.abs(exact))) - 8)
        worst = max(worst, float(((np.abs(o - exact) - half) / np.abs(exact) / (2.0 ** -24 * (10 + 2 * (t // 32)))).max()))
    assert worst <= 1


def decayed(g, n):
    """l^n in 64 bits, and how far c roundings of the state may be from it: each is off by half a unit at most and independent of the others (a step takes away 2^-12 of
    the state or more, and the next step's by a unit less), so that their sum has a spread of 2^-24 sqrt(c / 3), of which five; the exponent has a rounding or
    two (its share of n g each), a power as well."""
    g = g.astype(np.float64)
    return lambda c: (np.exp(n * g), 2.0 ** -24 * (5 * np.sqrt(c / 3) + 4 * np.abs(n * g) + 8))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("S,H,dh", [(131072, 257, 1), (131072, 2, 8)])
def test_a_state_decays_by_the_power_however_long_the_chain(K, dtype, S, H, dh):
    """Keys, values, queries and dout of zeros: s_out = l^S s0 and ds0 = l^S ds_out after 4096 chunks, one after another (many heads) or in segments."""
    import torch
    n = [K.lpk_linear_attention_scratch(1, S, H, dh, b) for b in (0, 1)]
    assert (max(n) == 0) == (H == 257)
    g = np.log1p(-np.exp2(-np.linspace(12, 17, H))).astype(np.float32)
    tdt = torch.bfloat16 if dtype else torch.float32
    qkv, dqkv = torch.zeros(S, 3 * H * dh, device="cuda", dtype=tdt), torch.ones(S, 3 * H * dh, device="cuda", dtype=tdt)
    o, dout = torch.ones(S, H * dh, device="cuda", dtype=tdt), torch.zeros(S, H * dh, device="cuda", dtype=tdt)
    s0 = 1 + torch.rand(1, H, dh, dh, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    s_out, ds0 = torch.empty_like(s0), torch.empty_like(s0)
    decay, ws = torch.from_numpy(g).cuda(), torch.empty(max(n) + 1, device="cuda")
    K.lpk_linear_attention_fwd(dtype, qkv, decay, None, s0, o, s_out, 1, S, H, dh, ws)
    # o_t = l^{t + 1} q_t s0 with q_t = 0; dq_t = 0 likewise
    K.lpk_linear_attention_bwd(dtype, qkv, decay, None, s0, dout, s0, dqkv, ds0, 1, S, H, dh, ws)
    want, tol = decayed(g, S)(S / 32)
    for got in (s_out, ds0):
        ratio = (got.double() / s0.double()).cpu().numpy().reshape(H, -1)
        assert (np.abs(ratio / want[:, None] - 1) <= tol[:, None]).all()
    assert not o.any() and not dqkv.any()


def test_a_state_decays_by_the_power_token_after_token(K):
    """8192 roundings, as above, but not independent at every decay: with m = 1 - l a step takes m s units away, the next one m^2 s 2^24 units less, that difference
    falls by m^3 s 2^24 = 0.94 units a step at m = 0.0038222, and near a whole number the same roundings come again and again (the recurrence rounded exactly, on the
    host: 2.75e-5 there, whatever the state begins with, and 2.0e-6 to 3.0e-6 as the root mean square over these decays; with l rounded instead 1.5e-4).
    So the root mean square over the decays counts, of which the spread above is one part: twice that is allowed; and n halves of a unit for each, which is all that
    can come together."""
    import torch
    H, n = 256, 8192
    g = np.log1p(-np.exp2(-np.linspace(8, 12, H))).astype(np.float32)
    decay = torch.from_numpy(g).cuda()
    s0 = 1 + torch.rand(1, H, 1, 1, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    state, qkv, o = s0.clone(), torch.zeros(1, 3 * H, device="cuda"), torch.empty(1, H, device="cuda")
    for _ in range(n):
        K.lpk_linear_attention_step(0, qkv, decay, state, o, 1, H, 1)
    want, tol = decayed(g, n)(n)
    off = np.abs((state.double() / s0.double()).cpu().numpy().reshape(H) / want - 1)
    assert np.sqrt((off ** 2).mean()) <= 2.0 ** -24 * (2 * np.sqrt(n / 3) + 4 * np.abs(n * g.astype(np.float64)).mean() + 8)
    assert (off <= tol + n * 2.0 ** -24).all()


# ------------------------------------------------------------------------------------------------ long axes, whatever the sizes
def cut_case(K, dtype, B, S, H, dh, **kw):
    """A case both directions of which are cut into segments."""
    assert all(K.lpk_linear_attention_scratch(B, S, H, dh, b) > 0 for b in (0, 1))
    return Case(dtype, B, S, H, dh, **kw)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dh", [1, 3, 8, 20, 33, 40, 72, 96, 100, 127])
def test_segments_of_all_head_sizes(K, dtype, dh):
    cut_case(K, dtype, 2, 640, 2, dh, seed=dh).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dh", [32, 64, 96, 128, 63])
@pytest.mark.parametrize("lens", [None, [640, 317]])
def test_segments_without_states(K, dtype, dh, lens):
    cut_case(K, dtype, 2, 640, 2, dh, seed=dh, states=False, lens=lens).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dh,states", [(64, True), (64, False), (96, True), (128, True), (21, True)])
def test_segments_of_unaligned_buffers(K, dtype, dh, states):
    cut_case(K, dtype, 2, 650, 2, dh, seed=6, states=states, shift=1).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("decay", [[0.0, 0.0], [-np.inf, -50.0], [-1e-4, -4.0]])
@pytest.mark.parametrize("lens", [None, [0, 641]])
def test_segments_of_decays_at_their_limits(K, dtype, decay, lens):
    cut_case(K, dtype, 2, 700, 2, 64, seed=5, decay=decay, lens=lens).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("states", [False, True])
def test_heads_of_96_uncut(K, dtype, states):
    assert K.lpk_linear_attention_scratch(2, 150, 2, 96, 1) == 0
    Case(dtype, 2, 150, 2, 96, seed=1, states=states).check(K)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("S,dh", [(130, 64), (130, 128), (600, 64), (600, 32), (640, 128)])
@pytest.mark.parametrize("which,value", [(0, np.inf), (0, np.nan), (1, -np.inf), (1, np.nan), (2, np.inf), (2, np.nan), (3, np.inf), (3, np.nan)])
def test_infinities_stay_to_the_end(K, dtype, S, dh, which, value):
    """q, k, v or dout with one bad column in one row: every output that has it in a sum is an infinity or a NaN, in later chunks and segments too."""
    at, col, H = 77, 5, 2
    case = Case(dtype, 1, S, H, dh, seed=4)
    (case.dout if which == 3 else case.qkv)[at, (0 if which == 3 else which * H * dh) + col] = value       # head 0
    d = case.upload()
    case.outputs()
    case.forward(K)
    case.backward(K)
    out = {n: d[n].float().cpu().numpy() for n in ("o", "dqkv")}
    w = H * dh
    outs = {"o": out["o"][:, :dh], **{n: out["dqkv"][:, i * w:i * w + dh] for i, n in enumerate(("dq", "dk", "dv"))}}
    every, one, before, here, after = slice(None), col, slice(0, at + 1), slice(at, at + 1), slice(at, S)
    bad = [dict(o=(here, every), dk=(before, one), dv=(before, every)), dict(o=(after, every), dq=(after, one), dv=(here, every)),
           dict(o=(after, one), dq=(after, every), dk=(here, every)), dict(dq=(here, every), dk=(before, every), dv=(before, one))][which]
    for n, where in bad.items():
        assert not np.isfinite(outs[n][where]).any(), n
    states = {0: d["ds0"], 1: d["s_out"], 2: d["s_out"], 3: d["ds0"]}[which].cpu().numpy()[0, 0]
    assert not np.isfinite(states[col] if which in (0, 1) else states[:, col]).any()
