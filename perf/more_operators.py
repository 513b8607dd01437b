"""What the operators of a decoder that answers token by token are measured on.

Three operators: rotary positions (training and single tokens), a paged cache of keys and values that is quantised to 8 bits as
it is written and read back, and attention over that cache (single tokens, prompts, chunks of prompts).  One pass is one call, or a
forward and a backward call of the rotary positions, on device buffers that the caller keeps, as a training or serving program makes them.

With `own` false the operators are computed in their plain form, elementary torch operations in 32 bits, angles in 64.

The cache: pages of `page` tokens, keys [pages, heads, page, dh] and values [pages, heads, dh, page] in e4m3, a scale (fp32, a power of two)
for every page and head; `table` [B, most pages] says which pages hold a sequence.  New rows of sequence b are rows starts[b] .. starts[b + 1]
of their matrix (row b where there is one for each) and the last positions of lens[b].
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"


# ------------------------------------------------------------------------------------------------ cases
def _rotary(**kw):
    return dict(dict(op="rotary", dtype=BF16, rows=1, heads=24, dh=64, rot=64, interleaved=False, far=1024, factor=1.0, train=False), **kw)


def _cache(op, **kw):
    return dict(dict(op=op, dtype=BF16, B=1, T=1, L=1024, ragged=False, H=12, Hkv=12, dh=64, page=64), **kw)


def listed():
    return [
        # Decoding for five users in fp32, deep in contexts that were stretched eightfold: pairs of neighbours, part of the head; latency.
        _rotary(name="rotary_step", dtype=F32, rows=5, heads=9, dh=80, rot=32, interleaved=True, far=1000003, factor=8.0),
        # Queries and keys of a layer of the twelve-layer decoder in training, forward and backward.
        _rotary(name="rotary_train", rows=8192, train=True),
        # Decoding for one user: one token of twelve heads goes into the cache; nothing but latency.
        _cache("append", name="append_step", L=777),
        # Decoding for many users: a token each, at all depths of their pages.
        _cache("append", name="append_batch", B=192, L=4096, ragged=True, H=16, Hkv=16),
        # Prompts of many lengths into the cache.
        _cache("append", name="append_prompt", B=8, T=2048, L=2048, ragged=True, H=32, Hkv=8, dh=128),
        # A session's cache back into tensors, to go on in training or to be written to a file.
        _cache("read", name="read_back", B=4, T=4096, L=4096, H=16, Hkv=16),
        # Odd lengths, a few heads and small pages, in fp32.
        _cache("read", name="read_back_odd", dtype=F32, B=3, T=511, L=1300, ragged=True, H=5, Hkv=5, dh=48, page=16),
        # One token for one user: latency.
        _cache("attention", name="attention_step", L=1000),
        # One token each for many users whose contexts have every length, four query heads to a head of the cache.
        _cache("attention", name="attention_step_batch", B=192, L=4096, ragged=True, H=32, Hkv=8, dh=128),
        # One token for two users over very long contexts: few heads, a long axis.
        _cache("attention", name="attention_step_long", B=2, L=131071, H=16, Hkv=4, page=128),
        # Prompts, right after they were written.
        _cache("attention", name="attention_prompt", B=8, T=4096, L=4096, ragged=True),
        # The next chunk of three long prompts in fp32: an odd number of rows over what is there already.
        _cache("attention", name="attention_chunk", dtype=F32, B=3, T=509, L=8000, ragged=True, H=8, Hkv=2, dh=96, page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["rotary", "append", "read", "attention", "attention", "attention"])
    dtype = rng.choice([BF16, BF16, F32])
    if op == "rotary":
        dh = rng.choice([16, 24, 32, 48, 64, 64, 80, 96, 128, 192])
        rot = rng.choice([dh, dh, 2 * rng.randint(1, dh // 2)])
        heads = rng.randint(1, 40)
        return _rotary(dtype=dtype, rows=_log_int(rng, 1, 2 ** 23 // (heads * dh)), heads=heads, dh=dh, rot=rot, interleaved=rng.random() < 0.5,
                       far=_log_int(rng, 64, 2 ** 21), factor=rng.choice([1.0, 1.0, 4.0, 32.0]), train=rng.random() < 0.6)
    Hkv, dh, page = rng.randint(1, 16), rng.choice([16, 32, 48, 64, 64, 80, 96, 128, 128, 192, 256]), rng.choice([16, 32, 64, 64, 128, 256])
    H = Hkv * (rng.choice([1, 2, 3, 4, 8]) if op == "attention" else 1)
    geometry = dict(dtype=dtype, ragged=rng.random() < 0.6, H=H, Hkv=Hkv, dh=dh, page=page)
    if op != "attention":
        n = 2 ** 24 // (Hkv * dh)                # new rows in all, at most
        T = rng.choice([1, _log_int(rng, 1, min(n, 4096))])
        B = _log_int(rng, 1, max(1, min(n // T, 256)))
        return _cache(op, B=B, T=T, L=_log_int(rng, T, max(T, min(16384, 2 ** 28 // (B * Hkv * dh)))), **geometry)
    T = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 2048)])
    # what is read, and what is computed: at most 0.4 GB and 60 GFLOP (a few rows' own tensors and a whole prompt's later half aside)
    T = min(T, int(math.sqrt(1.5e10 / (H * dh))))
    most = min(2e8 / (Hkv * dh), 1.5e10 / (H * dh * T))
    L = _log_int(rng, T, max(T, min(most, 131072)))
    return _cache(op, B=_log_int(rng, 1, max(1, min(int(most // L), 256))), T=T, L=L, **geometry)


def _spread(c):
    """(length, new rows) of every sequence, in order: the longest has L and T, and where they are ragged the others less, down to a
    single token and a row."""
    B, T, L = c["B"], c["T"], c["L"]
    if not c["ragged"]:
        return [(L, T)] * B
    lens = [max(1, (L * (B - b)) // B) for b in range(B)]
    return [(n, min(n, max(1, T - (b * T) // (2 * B)))) for b, n in enumerate(lens)]


def work(case):
    c = case
    e = 2 if c["dtype"] == BF16 else 4
    if c["op"] == "rotary":
        n = c["rows"] * c["heads"] * c["dh"] * (2 if c["train"] else 1)
        return {"bytes": 2 * e * n + 4 * c["rows"], "flops": 3.0 * n * c["rot"] / c["dh"]}
    both = _spread(c)
    rows, tokens, w = sum(n for _, n in both), sum(n for n, _ in both), c["Hkv"] * c["dh"]
    if c["op"] == "attention":
        pairs = sum(n * (2 * ln - n + 1) / 2 for ln, n in both)
        return {"bytes": 2 * w * tokens + 8 * c["Hkv"] * tokens / c["page"] + rows * c["H"] * (2 * e * c["dh"] + 4), "flops": 4.0 * pairs * c["H"] * c["dh"]}
    return {"bytes": 2 * rows * w * (e + 1) + 8 * c["Hkv"] * rows / c["page"], "flops": 4.0 * rows * w}


# ------------------------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == BF16 else torch.float32


def _frequencies(rot, factor):
    """Radians a position; stretched ones divide by `factor` what turns less than once in 4096 positions, keep what turns 32 times, and
    go from one to the other between."""
    f = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    kept = np.clip((4096 * f / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
    return f * (kept + (1.0 - kept) / factor)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T_ = _dt(c)

    def normal(*shape, scale=1.0, dtype=None):
        return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(dtype or T_)

    def room(*shape, dtype=None):
        return torch.empty(*shape, device="cuda", dtype=dtype or T_)

    st = {"case": c, "code": 1 if c["dtype"] == BF16 else 0}
    if c["op"] == "rotary":
        rows, n = c["rows"], c["heads"] * c["dh"]
        # the rotated heads are the front part of a wider row: queries and keys with the values behind them
        st["x"] = normal(rows, n + n // 2)[:, :n]
        st["pos"] = torch.randint(0, c["far"], (rows,), device="cuda", generator=gen, dtype=torch.int32)
        st["freq"] = torch.from_numpy(_frequencies(c["rot"], c["factor"])).cuda()
        st["scale"] = 1.0 + 0.1 * math.log(c["factor"])        # the length of stretched queries and keys
        st["y"] = room(rows, n)
        if c["train"]:
            st["dy"], st["dx"] = normal(rows, n, scale=1.0 / 64), room(rows, n)
        return st
    B, T, Hkv, dh, P = (c[k] for k in ("B", "T", "Hkv", "dh", "page"))
    both = _spread(c)
    random.Random(seed).shuffle(both)
    st["lens"] = torch.tensor([n for n, _ in both], dtype=torch.int32).cuda()
    rows = sum(n for _, n in both)
    st["starts"] = None if rows == B * T else torch.tensor(np.cumsum([0] + [n for _, n in both]), dtype=torch.int32).cuda()
    # pages of a pool in which sequences come and go: in no order, some of them nobody's
    most = -(-c["L"] // P)
    pages = B * most + 3
    st["table"] = torch.randperm(pages, device="cuda", generator=gen)[:B * most].to(torch.int32).reshape(B, most)
    st["kpages"] = torch.empty(pages, Hkv, P, dh, device="cuda", dtype=torch.float8_e4m3fn)
    st["vpages"] = torch.empty(pages, Hkv, dh, P, device="cuda", dtype=torch.float8_e4m3fn)
    for pool in (st["kpages"], st["vpages"]):
        for i in range(0, pages, 4096):
            part = pool[i:i + 4096]
            part.copy_(normal(*part.shape, scale=64.0, dtype=torch.float32).clamp_(-448.0, 448.0))
    for name in ("kscale", "vscale"):
        st[name] = torch.exp2(torch.randint(-7, -4, (pages, Hkv), device="cuda", generator=gen).float())
    if c["op"] == "append":
        # keys and values as the projection leaves them, side by side
        kv = normal(rows, 2 * Hkv * dh)
        st["k"], st["v"] = kv[:, :Hkv * dh], kv[:, Hkv * dh:]
    elif c["op"] == "read":
        st["k"], st["v"] = room(rows, Hkv * dh), room(rows, Hkv * dh)
    else:
        H = c["H"]
        st["q"] = normal(rows, (H + 2 * Hkv) * dh)[:, :H * dh]
        st["o"], st["lse"] = room(rows, H * dh), room(rows, H, dtype=torch.float32)
        st["scratch"] = {}                       # what a single call may use as workspace, kept by the program
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    return (_own if own else _plain)[st["case"]["op"]](st)


def _own_rotary(st):
    from paper_2012_03837_amd import kernels as K
    c = st["case"]
    how = (c["rows"], 1, c["heads"], c["dh"], c["rot"], int(c["interleaved"]), st["scale"])
    K.lpk_rotary(st["code"], st["x"], st["y"], st["pos"], st["freq"], *how)
    if not c["train"]:
        return {"y": st["y"]}
    K.lpk_rotary(st["code"], st["dy"], st["dx"], st["pos"], st["freq"], *how, backward=1)
    return {"y": st["y"], "dx": st["dx"]}


def _paged(st):
    return (st["starts"], st["lens"], st["table"], st["kpages"], st["vpages"], st["kscale"], st["vscale"])


def _own_append(st):
    from paper_2012_03837_amd import kernels as K
    c = st["case"]
    K.lpk_cache_append(st["code"], st["k"], st["v"], *_paged(st), c["B"], c["T"], c["Hkv"], c["dh"], c["page"])
    return {n: st[n] for n in ("kpages", "vpages", "kscale", "vscale")}


def _own_read(st):
    from paper_2012_03837_amd import kernels as K
    c = st["case"]
    K.lpk_cache_read(st["code"], st["k"], st["v"], *_paged(st), c["B"], c["T"], c["Hkv"], c["dh"], c["page"])
    return {"k": st["k"], "v": st["v"]}


def _own_attention(st):
    from paper_2012_03837_amd import kernels as K
    c = st["case"]
    size = tuple(c[k] for k in ("B", "T", "H", "Hkv", "dh", "page"))
    if "ws" not in st["scratch"]:
        floats = K.lpk_cache_attention_scratch(*size, st["table"].shape[1])
        st["scratch"]["ws"] = torch.empty(max(1, floats), device="cuda", dtype=torch.float32)
    K.lpk_cache_attention(st["code"], st["q"], *_paged(st), st["o"], st["lse"], *size, 1, st["scratch"]["ws"])
    return {"o": st["o"], "lse": st["lse"]}


def _plain_rotate(x, st, back):
    c = st["case"]
    rot, half = c["rot"], c["rot"] // 2
    angle = st["pos"].double()[:, None] * st["freq"]
    cos, sin = (f(angle).float()[:, None, :] * st["scale"] for f in (torch.cos, torch.sin))
    if back:
        sin = -sin
    x = x.float().reshape(c["rows"], c["heads"], c["dh"])
    y = x.clone()
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, half), slice(half, rot))
    a, b = x[..., one], x[..., two]
    y[..., one], y[..., two] = a * cos - b * sin, a * sin + b * cos
    return y.reshape(c["rows"], -1).to(_dt(c))


def _plain_rotary(st):
    out = {"y": _plain_rotate(st["x"], st, False)}
    if st["case"]["train"]:
        out["dx"] = _plain_rotate(st["dy"], st, True)
    return out


def _places(st):
    """Of every new row its page and its place there, and the pages that new rows stand in (some of them several times)."""
    c = st["case"]
    B, T = c["B"], c["T"]
    lens = st["lens"].long()
    rows = st["k"].shape[0]
    starts = torch.arange(B + 1, device="cuda") * T if st["starts"] is None else st["starts"].long()
    row = torch.arange(rows, device="cuda")
    b = torch.searchsorted(starts, row, right=True) - 1
    pos = lens[b] - (starts[b + 1] - row)
    table, P = st["table"].long(), c["page"]
    slot = (lens - starts[1:] + starts[:-1])[:, None] // P + torch.arange((T + P - 2) // P + 1, device="cuda")
    return table[b, pos // P], pos % P, table.gather(1, torch.minimum(slot, (lens[:, None] - 1) // P)).reshape(-1)


def _plain_append(st):
    c = st["case"]
    Hkv, dh, P = c["Hkv"], c["dh"], c["page"]
    page, at, hit = _places(st)
    pages = st["kpages"].shape[0]
    first = torch.full((pages,), P, device="cuda").scatter_reduce(0, page, at, "amin")
    first = torch.where(first < P, first, 0)                  # how many earlier tokens a page that is written to has
    for x, pool, scale, dims in ((st["k"], st["kpages"], st["kscale"], (2, 3)), (st["v"], st["vpages"], st["vscale"], (3, 2))):
        x = x.float().reshape(-1, Hkv, dh)
        most = torch.zeros(pages, Hkv, device="cuda").scatter_reduce(0, page[:, None].expand(-1, Hkv), x.abs().amax(2), "amax")
        m, e = torch.frexp(most)
        need = torch.where(most > 0, torch.ldexp(torch.ones_like(most), torch.where(m <= 0.875, e - 9, e - 8)), 2.0 ** -126)
        new = torch.maximum(torch.where(first[:, None] > 0, scale, 0.0), need)
        old = pool.view(torch.uint8)[hit].view(torch.float8_e4m3fn).float()
        ratio = (scale[hit] / new[hit])[:, :, None, None]
        earlier = torch.arange(P, device="cuda")[None, :] < first[hit][:, None]
        earlier = earlier[:, None, :, None] if dims[0] == 2 else earlier[:, None, None, :]
        old = torch.where(earlier, old * ratio, old).to(torch.float8_e4m3fn)
        pool.view(torch.uint8)[hit] = old.view(torch.uint8)
        code = (x / new[page][:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        if dims[0] == 2:
            pool.view(torch.uint8)[page, :, at] = code
        else:
            pool.view(torch.uint8)[page, :, :, at] = code
        scale[hit] = new[hit]
    return {n: st[n] for n in ("kpages", "vpages", "kscale", "vscale")}


def _plain_read(st):
    c = st["case"]
    page, at, _ = _places(st)
    k = st["kpages"].view(torch.uint8)[page, :, at].view(torch.float8_e4m3fn).float() * st["kscale"][page][:, :, None]
    v = st["vpages"].view(torch.uint8)[page, :, :, at].view(torch.float8_e4m3fn).float() * st["vscale"][page][:, :, None]
    return {"k": k.reshape(k.shape[0], -1).to(_dt(c)), "v": v.reshape(v.shape[0], -1).to(_dt(c))}


def _plain_attention(st):
    c = st["case"]
    B, T, H, Hkv, dh, P = (c[k] for k in ("B", "T", "H", "Hkv", "dh", "page"))
    G, rows, S = H // Hkv, st["q"].shape[0], st["table"].shape[1] * P
    lens = st["lens"].long()
    starts = torch.arange(B + 1, device="cuda") * T if st["starts"] is None else st["starts"].long()
    q = st["q"].float().reshape(rows, Hkv, G, dh)
    o, lse = torch.zeros(rows + 1, H, dh, device="cuda"), torch.zeros(rows + 1, H, device="cuda")
    step = max(1, min(B, 2 ** 28 // (S * max(Hkv * dh, H * T))))
    t, key = torch.arange(T, device="cuda"), torch.arange(S, device="cuda")
    for b in range(0, B, step):
        part = slice(b, b + step)
        table, ln, first = st["table"][part].long(), lens[part], starts[:-1][part]
        n, g = starts[1:][part] - first, table.shape[0]
        k = st["kpages"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * st["kscale"][table][..., None, None]
        k = k.permute(0, 2, 1, 3, 4).reshape(g, Hkv, S, dh)
        v = st["vpages"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * st["vscale"][table][..., None, None]
        v = v.permute(0, 2, 1, 4, 3).reshape(g, Hkv, S, dh)
        row = torch.where(t < n[:, None], first[:, None] + t, rows)                     # those that are not there go into one more row
        qs = q[row.clamp(max=rows - 1)].permute(0, 2, 3, 1, 4).reshape(g, Hkv, G * T, dh)
        s = (qs @ k.transpose(-1, -2)).reshape(g, Hkv, G, T, S) / math.sqrt(dh)
        last = ln[:, None] - n[:, None] + t                                            # a row's own position
        seen = (key <= last[:, :, None])[:, None, None]
        s = torch.where(seen, s, float("-inf"))
        top = s.amax(-1, keepdim=True)
        top = torch.where(top > float("-inf"), top, 0.0)
        w = torch.exp(s - top)
        total = w.sum(-1, keepdim=True)
        out = (w.reshape(g, Hkv, G * T, S) @ v).reshape(g, Hkv, G, T, dh) / total
        o[row] = out.permute(0, 3, 1, 2, 4).reshape(g, T, H, dh)
        lse[row] = (top + torch.log(total)).permute(0, 3, 1, 2, 4).reshape(g, T, H)
    return {"o": o[:rows].reshape(rows, H * dh).to(_dt(c)), "lse": lse[:rows]}


_own = dict(rotary=_own_rotary, append=_own_append, read=_own_read, attention=_own_attention)
_plain = dict(rotary=_plain_rotary, append=_plain_append, read=_plain_read, attention=_plain_attention)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        out = {"y": _exact_rotary(st, st["x"], 1.0)}
        if case["train"]:
            out["dx"] = _exact_rotary(st, st["dy"], -1.0)
        return out
    return dict(append=_exact_append, read=_exact_read, attention=_exact_attention)[case["op"]](st)


def _exact_rotary(st, x, turn):
    """Pairs as complex numbers, turned by their angle."""
    c = st["case"]
    rot = c["rot"]
    x = x.double().reshape(c["rows"], c["heads"], c["dh"])
    front, rest = x[..., :rot], x[..., rot:]
    pairs = front.reshape(*front.shape[:2], rot // 2, 2) if c["interleaved"] else front.reshape(*front.shape[:2], 2, rot // 2).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous())
    angle = turn * st["pos"].double().unsqueeze(1) * st["freq"].unsqueeze(0)
    z = torch.view_as_real(z * torch.polar(torch.full_like(angle, st["scale"]), angle).unsqueeze(1))
    front = z.reshape(front.shape) if c["interleaved"] else z.transpose(-1, -2).reshape(front.shape)
    return torch.cat([front, rest], -1).reshape(c["rows"], -1)


def _sequences(st):
    """(first row, rows, length, pages) of every sequence, on the host."""
    c = st["case"]
    starts = [b * c["T"] for b in range(c["B"] + 1)] if st["starts"] is None else st["starts"].tolist()
    return [(starts[b], starts[b + 1] - starts[b], n, st["table"][b].tolist()) for b, n in enumerate(st["lens"].tolist())]


def _exact_append(st):
    """Page by page; what is held in 8 bits stands there before its rounding."""
    c = st["case"]
    Hkv, dh, P = c["Hkv"], c["dh"], c["page"]
    out = {}
    for name, x, pool, scale, turned in (("k", st["k"], st["kpages"], st["kscale"], False), ("v", st["v"], st["vpages"], st["vscale"], True)):
        x = x.double().reshape(-1, Hkv, dh)
        held = pool.float().double()
        held = held.transpose(2, 3).contiguous() if turned else held
        scale = scale.double().clone()
        for first, n, length, pages in _sequences(st):
            for slot in range((length - n) // P, -(-length // P)):
                lo, hi = max(0, length - n - slot * P), min(P, length - slot * P)
                new = x[first + slot * P + lo - (length - n):first + slot * P + hi - (length - n)]
                p = pages[slot]
                need = torch.exp2(torch.ceil(torch.log2(new.abs().amax((0, 2)) / 448.0)))
                s = torch.maximum(need, scale[p]) if lo > 0 else need
                held[p, :, :lo] *= (scale[p] / s).reshape(Hkv, 1, 1)
                held[p, :, lo:hi] = (new / s.reshape(1, Hkv, 1)).transpose(0, 1)
                scale[p] = s
        out[name + "pages"] = held.transpose(2, 3).contiguous() if turned else held
        out[name + "scale"] = scale
    return {n: out[n] for n in ("kpages", "vpages", "kscale", "vscale")}


def _tokens(st, pages, lo, hi):
    """Keys and values of positions lo .. hi - 1 of a sequence, [heads, positions, dh] in 64 bits."""
    P = st["case"]["page"]
    ids = torch.tensor(pages, device="cuda")[lo // P:-(-hi // P)]
    k = st["kpages"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * st["kscale"][ids].double().reshape(*st["kscale"][ids].shape, 1, 1)
    v = st["vpages"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * st["vscale"][ids].double().reshape(*st["vscale"][ids].shape, 1, 1)
    cut = slice(lo - lo // P * P, lo - lo // P * P + hi - lo)
    k = k.transpose(0, 1).reshape(k.shape[1], -1, k.shape[3])
    v = v.permute(1, 0, 3, 2).reshape(v.shape[1], -1, v.shape[2])
    return k[:, cut], v[:, cut]


def _exact_read(st):
    k, v = st["k"].double(), st["v"].double()
    for first, n, length, pages in _sequences(st):
        a, b = _tokens(st, pages, length - n, length)
        k[first:first + n], v[first:first + n] = a.transpose(0, 1).reshape(n, -1), b.transpose(0, 1).reshape(n, -1)
    return {"k": k, "v": v}


def _exact_attention(st):
    """From the definition, one sequence and head of the cache at a time."""
    c = st["case"]
    H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
    G = H // Hkv
    rows = st["q"].shape[0]
    q = st["q"].double().reshape(rows, H, dh)
    o, lse = torch.zeros(rows, H, dh, device="cuda", dtype=torch.float64), torch.zeros(rows, H, device="cuda", dtype=torch.float64)
    for first, n, length, pages in _sequences(st):
        k, v = _tokens(st, pages, 0, length)
        own_place = torch.arange(length - n, length, device="cuda")
        hidden = torch.arange(length, device="cuda").unsqueeze(0) > own_place.unsqueeze(1)
        for h in range(H):
            if h % G == 0:
                kt, vh = k[h // G].t().contiguous(), v[h // G].contiguous()
            s = torch.mm(q[first:first + n, h].contiguous(), kt) * dh ** -0.5
            if n > 1:
                s.masked_fill_(hidden, float("-inf"))
            lse[first:first + n, h] = torch.logsumexp(s, 1)
            o[first:first + n, h] = torch.mm(torch.softmax(s, 1), vh)
    return {"o": o.reshape(rows, H * dh), "lse": lse}
