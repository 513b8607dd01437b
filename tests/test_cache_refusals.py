"""What the entry points of rotary positions and the 8-bit cache refuse, on the host: every call here ends before anything is launched (the
addresses are not memory)."""
import pytest

P, NULL = 1 << 20, None            # never read


@pytest.fixture(scope="module")
def K():
    from paper_2012_03837_amd import kernels
    return kernels


def call(K, name, **kw):
    args = DEFAULTS[name] | kw
    assert set(args) == set(DEFAULTS[name])
    return K._fn(name)(*args.values(), None)


PAGED = dict(starts=P, lens=P, table=P, kpages=P, vpages=P, kscale=P, vscale=P)
SIZE = dict(page=64, max_pages=5, n_pages=20)
ROWS = dict(dtype=1, k=P, ldk=256, v=P, ldv=256, rows=30, **PAGED, B=3, T=10, Hkv=4, dh=64, **SIZE)
DEFAULTS = {
    "lpk_rotary": dict(dtype=1, x=P, ldx=256, y=P, ldy=256, pos=P, freq=P, rows=30, S=1, heads=4, dh=64, rot=32, interleaved=0, scale=1.0, backward=0),
    "lpk_cache_append": ROWS, "lpk_cache_read": ROWS,
    "lpk_cache_attention": dict(dtype=1, q=P, ldq=512, rows=30, **PAGED, o=2 * P, ldo=512, lse=P, B=3, T=10, H=8, Hkv=4, dh=64, **SIZE, causal=1, scratch=P,
                                elems=1 << 26),
}
CACHE = [dict(dtype=2), dict(dtype=-1), dict(B=-1), dict(B=(1 << 20) + 1), dict(T=0), dict(T=-1), dict(rows=-1), dict(Hkv=0), dict(dh=0), dict(dh=8), dict(dh=72), dict(dh=272),
         dict(page=8), dict(page=48), dict(page=512), dict(page=0), dict(max_pages=0), dict(n_pages=0), dict(max_pages=1 << 25), dict(lens=NULL), dict(table=NULL),
         dict(kpages=NULL), dict(vpages=NULL), dict(kscale=NULL), dict(vscale=NULL), dict(kpages=P + 8), dict(vpages=P + 1), dict(starts=NULL, rows=29)]
BAD = {
    "lpk_rotary": [dict(dtype=2), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(S=0), dict(heads=0), dict(dh=0), dict(dh=513), dict(rot=0), dict(rot=33), dict(rot=66),
                   dict(heads=1 << 20, ldx=1 << 30, ldy=1 << 30), dict(ldx=255), dict(ldy=255), dict(ldx=1 << 33), dict(x=NULL), dict(y=NULL), dict(freq=NULL), dict(ldx=512)],
    "lpk_cache_append": CACHE + [dict(k=NULL), dict(v=NULL), dict(ldk=255), dict(ldv=255), dict(ldk=1 << 33), dict(Hkv=4097, ldk=1 << 20, ldv=1 << 20)],
    "lpk_cache_read": CACHE + [dict(k=NULL), dict(v=NULL), dict(ldk=255), dict(ldv=255)],
    "lpk_cache_attention": CACHE + [dict(q=NULL), dict(o=NULL), dict(ldq=511), dict(ldo=511), dict(H=6, ldq=384, ldo=384), dict(H=2), dict(H=0), dict(T=1 << 24, H=512, ldq=1 << 20, ldo=1 << 20)],
}


@pytest.mark.parametrize("name,kw", [(n, kw) for n in BAD for kw in BAD[n]], ids=str)
def test_refused(K, name, kw):
    assert call(K, name, **kw) == 1          # hipErrorInvalidValue


@pytest.mark.parametrize("name", DEFAULTS)
def test_nothing_to_do(K, name):
    assert call(K, name, rows=0) == 0
    if "B" in DEFAULTS[name]:
        assert call(K, name, B=0) == 0


def test_attention_workspace(K):
    """Short axes need none; a long one of few rows does, and a call without it is refused."""
    assert K.lpk_cache_attention_scratch(4, 1, 8, 8, 64, 64, 2) == 0
    n = K.lpk_cache_attention_scratch(1, 1, 8, 8, 64, 64, 1000)
    assert n > 0 and K.lpk_cache_attention_scratch(0, 1, 8, 8, 64, 64, 1000) == 0
    long = dict(B=1, T=1, rows=1, H=8, Hkv=8, ldq=512, ldo=512, max_pages=1000)
    for kw in (dict(scratch=NULL), dict(elems=n - 1), dict(scratch=P + 4)):
        assert call(K, "lpk_cache_attention", **(long | dict(elems=n) | kw)) == 1
    for kw in (dict(dh=40), dict(page=20), dict(H=7), dict(T=0), dict(B=-1)):
        assert K.lpk_cache_attention_scratch(*(dict(B=1, T=1, H=8, Hkv=8, dh=64, page=64, max_pages=1000) | kw).values()) == 0


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=3), dict(rot=-2), dict(base=0.0), dict(base=float("inf")), dict(base=float("nan")), dict(factor=0.0), dict(factor=-1.0), dict(factor=float("nan")),
                                dict(low=2.0, high=1.0), dict(low=float("nan")), dict(context=-1.0), dict(context=float("nan"))], ids=str)
def test_frequencies_refused(K, kw):
    with pytest.raises(K.KernelError):
        K.lpk_rotary_frequencies(**(dict(rot=8) | kw))


# ------------------------------------------------------------------------------------------------ the wrappers' own checks
# Tensors of the host: what is right but for that is refused for it last, everything else by its own check before.
B_, T_, H_, KV_, D_, P_, M_, N_, R_ = 3, 2, 4, 2, 16, 16, 4, 9, 6
_PAGED = dict(starts=("i", (B_ + 1,)), lens=("i", (B_,)), table=("i", (B_, M_)), kpages=("q", (N_, KV_, P_, D_)), vpages=("q", (N_, KV_, D_, P_)), kscale=("f", (N_, KV_)),
              vscale=("f", (N_, KV_)))
_ROWS = dict(dtype=(None, 1), k=("e", (R_, KV_ * D_)), v=("e", (R_, KV_ * D_)), **_PAGED, B=(None, B_), T=(None, T_), Hkv=(None, KV_), dh=(None, D_), page=(None, P_))
WRAPPED = {
    "lpk_rotary": dict(dtype=(None, 1), x=("e", (R_, H_ * D_)), y=("e", (R_, H_ * D_)), pos=("i", (R_,)), freq=("d", (D_ // 2,)), rows=(None, R_), S=(None, 1),
                       heads=(None, H_), dh=(None, D_), rot=(None, D_)),
    "lpk_cache_append": _ROWS, "lpk_cache_read": _ROWS,
    "lpk_cache_attention": dict(dtype=(None, 1), q=("e", (R_, H_ * D_)), **_PAGED, o=("e", (R_, H_ * D_)), lse=("f", (R_, H_)), B=(None, B_), T=(None, T_), H=(None, H_),
                                Hkv=(None, KV_), dh=(None, D_), page=(None, P_), causal=(None, 1), scratch=("f", (7,))),
}
OPERANDS = [(n, a) for n, args in WRAPPED.items() for a, (t, _) in args.items() if t]


def tensors(name):
    import torch
    types = dict(e=torch.bfloat16, f=torch.float32, i=torch.int32, q=torch.float8_e4m3fn, d=torch.float64)
    return {n: torch.zeros(size, dtype=types[t]) if t else size for n, (t, size) in WRAPPED[name].items()}


def refused(K, name, args, match):
    with pytest.raises(K.KernelError, match=match):
        getattr(K, name)(*args.values())


@pytest.mark.parametrize("name", WRAPPED)
def test_wrappers_reach_the_device_check(K, name):
    args = tensors(name)
    refused(K, name, args, "tensors on the host")
    refused(K, name, args | dict(dtype=2), "dtype 2")
    first = next(a for n, a in OPERANDS if n == name)
    refused(K, name, args | {first: None}, "no tensor")


@pytest.mark.parametrize("name,arg", OPERANDS)
def test_wrappers_refuse_tensors_of_another_type(K, name, arg):
    import torch
    args = tensors(name)
    other = {1: torch.int8, 2: torch.float16, 4: torch.float32 if args[arg].dtype == torch.int32 else torch.int32, 8: torch.int64}[args[arg].itemsize]
    for dt in (other, torch.float32 if args[arg].itemsize == 8 else torch.float64):
        refused(K, name, args | {arg: args[arg].to(dt)}, "needed")


@pytest.mark.parametrize("name,arg", [x for x in OPERANDS if x[1] not in ("scratch", "table", "kpages")])
def test_wrappers_refuse_tensors_that_are_too_small(K, name, arg):
    import torch
    args = tensors(name)
    if arg in ("x", "y", "q", "o", "k", "v"):
        first = next(a for n, a in OPERANDS if n == name)
        if arg != first or name == "lpk_rotary":                              # the first matrix says how many rows there are
            refused(K, name, args | {arg: args[arg][:-1]}, "matrix of at least")
        refused(K, name, args | {arg: args[arg][:, :-1]}, "matrix of at least")
        refused(K, name, args | {arg: args[arg].reshape(-1)}, "matrix of at least")
        refused(K, name, args | {arg: args[arg].repeat(1, 2)[:, ::2]}, "contiguous")
        refused(K, name, args | {arg: args[arg][:1].expand(args[arg].shape)}, "contiguous")
        refused(K, name, args | {arg: args[arg].repeat(1, 3)[:, 5:5 + args[arg].shape[1]]}, "tensors on the host")
        return
    flat = args[arg].reshape(-1)
    refused(K, name, args | {arg: flat[:-1]}, "contiguous")
    refused(K, name, args | {arg: torch.cat([flat, flat])}, "tensors on the host")
    refused(K, name, args | {arg: torch.cat([flat, flat])[::2]}, "contiguous")


def test_pools_and_tables_go_by_their_sizes(K):
    """Fewer pages of keys are fewer pages; a table that is no whole number of rows leaves its last entries out."""
    for name in ("lpk_cache_append", "lpk_cache_read", "lpk_cache_attention"):
        args = tensors(name)
        refused(K, name, args | dict(kpages=args["kpages"][:-1]), "tensors on the host")
        refused(K, name, args | dict(kpages=args["kpages"].repeat(2, 1, 1, 1)), "contiguous")      # more than the others hold
        refused(K, name, args | dict(table=args["table"].reshape(-1)[:-1]), "tensors on the host")
        for arg in ("B", "T", "Hkv", "dh", "page"):
            with pytest.raises(K.KernelError):
                getattr(K, name)(*(args | {arg: args[arg] + (1 << 32)}).values())


def test_wrappers_refuse_numbers_that_would_wrap(K):
    for name, arg in (("lpk_rotary", "S"), ("lpk_cache_append", "T"), ("lpk_cache_read", "T"), ("lpk_cache_attention", "T")):
        args = tensors(name)
        refused(K, name, args | {arg: args[arg] + (1 << 32)}, "31 bits")
        refused(K, name, args | {arg: -1}, "31 bits")
