"""ctypes binding of the kernel-level ABI (include/lp_kernels.h): argument marshalling only.
Arguments are torch CUDA tensors (or None); every function enqueues on torch's current stream."""
from __future__ import annotations

import ctypes as C

from .binding import lib


class KernelError(RuntimeError):
    pass


def _p(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ck(rc, what):
    if rc != 0:
        raise KernelError(f"{what} failed with hipError {rc}")


_i, _i64, _f, _sz = C.c_int, C.c_int64, C.c_float, C.c_size_t


def lpk_gemm(dtype, A, lda, a_kc, B, ldb, b_kc, Cout, ldc, c_f32, M, N, K, bias=None, act=0, pre=None, dact_src=None,
             dact=0, ldd=0, res=None, ldr=0, accumulate=0, plain=0, splitk_ws=None, variant=None):
    variant = (1 if plain else 0) if variant is None else variant
    _ck(lib().lpk_gemm(_i(dtype), _p(A), _i64(lda), _i(a_kc), _p(B), _i64(ldb), _i(b_kc), _p(Cout), _i64(ldc),
                       _i(c_f32), _i(M), _i(N), _i(K), _p(bias), _i(act), _p(pre), _p(dact_src), _i(dact), _i64(ldd),
                       _p(res), _i64(ldr), _i(accumulate), _i(variant), _p(splitk_ws),
                       _sz(0 if splitk_ws is None else splitk_ws.numel()), _stream()), "lpk_gemm")


def lpk_gemm_grouped(As, Bs, Cs, Ms, Ns, K, a_kc, b_kc, accumulate, splitk_ws, biases=None, act=0, ress=None, tiles=None):
    """As, Bs, Cs: lists of torch CUDA tensors (bf16 operands as stored; outputs [M_i, N_i], all fp32 or all bf16);
    biases / ress: optional lists of fp32 [N_i] / bf16 [M_i, N_i] tensors; tiles: (shape, pieces) of lpk_gemm_grouped_tiles."""
    import torch
    n = len(As)
    vp = (C.c_void_p * n)
    i64 = (C.c_int64 * n)
    ia = (C.c_int * n)
    c_f32 = 1 if Cs[0].dtype == torch.float32 else 0
    bias = vp(*[b.data_ptr() for b in biases]) if biases is not None else None
    res = vp(*[r.data_ptr() for r in ress]) if ress is not None else None
    args = [_i(n), vp(*[a.data_ptr() for a in As]), i64(*[a.shape[1] for a in As]), vp(*[b.data_ptr() for b in Bs]),
            i64(*[b.shape[1] for b in Bs]), vp(*[c.data_ptr() for c in Cs]), i64(*[c.shape[1] for c in Cs]), _i(c_f32),
            ia(*Ms), ia(*Ns), _i(K), _i(a_kc), _i(b_kc), bias, _i(act), res, _i(accumulate), _p(splitk_ws),
            _sz(splitk_ws.numel()), _stream()]
    if tiles is None:
        _ck(lib().lpk_gemm_grouped(*args), "lpk_gemm_grouped")
    else:
        _ck(lib().lpk_gemm_grouped_tiles(_i(tiles[0]), _i(tiles[1]), *args), "lpk_gemm_grouped_tiles")


def lpk_weight_grads(dys, xs, dws, dbs, accumulate=0, splitk_ws=None, part=None, out=None, tiles=(-1, 1)):
    """dys [rows, M_i], xs [rows, N_i] (bf16), dws [M_i, N_i], dbs [M_i] or None (fp32); part [nblk, len] and out [len], or None."""
    n, vp = len(dys), C.c_void_p * len(dys)
    i64, ia = C.c_int64 * n, C.c_int * n
    ptr = lambda t: 0 if t is None else t.data_ptr()
    nblk, ln = (0, 0) if part is None else part.shape
    _ck(lib().lpk_weight_grads(_i(tiles[0]), _i(tiles[1]), _i(n), vp(*map(ptr, dys)), i64(*[d.shape[1] for d in dys]),
                               vp(*map(ptr, xs)), i64(*[x.shape[1] for x in xs]), vp(*map(ptr, dws)), vp(*map(ptr, dbs)),
                               ia(*[w.shape[0] for w in dws]), ia(*[w.shape[1] for w in dws]), _i(dys[0].shape[0]), _i(accumulate),
                               _p(part), _p(out), _i(nblk), _i(ln), _p(splitk_ws),
                               _sz(0 if splitk_ws is None else splitk_ws.numel()), _stream()), "lpk_weight_grads")


def lpk_attention_fwd(dtype, qkv, o, lse, B, S, H, dh, causal=1, plain=0):
    _ck(lib().lpk_attention_fwd(_i(dtype), _p(qkv), _p(o), _p(lse), _i(B), _i(S), _i(H), _i(dh), _i(causal), _i(plain),
                                _stream()), "lpk_attention_fwd")


def lpk_attention_bwd(dtype, qkv, o, lse, dout, dqkv, delta, B, S, H, dh, causal=1, plain=0):
    _ck(lib().lpk_attention_bwd(_i(dtype), _p(qkv), _p(o), _p(lse), _p(dout), _p(dqkv), _p(delta), _i(B), _i(S), _i(H),
                                _i(dh), _i(causal), _i(plain), _stream()), "lpk_attention_bwd")


def lpk_attention_fwd_parts(qkv, o, lse, B, S, H, dh, causal, parts):
    _ck(lib().lpk_attention_fwd_parts(_p(qkv), _p(o), _p(lse), _i(B), _i(S), _i(H), _i(dh), _i(causal), _i(parts), _stream()),
        "lpk_attention_fwd_parts")


def lpk_attention_bwd_parts(qkv, o, lse, dout, dqkv, delta, B, S, H, dh, causal, parts):
    _ck(lib().lpk_attention_bwd_parts(_p(qkv), _p(o), _p(lse), _p(dout), _p(dqkv), _p(delta), _i(B), _i(S), _i(H), _i(dh),
                                      _i(causal), _i(parts), _stream()), "lpk_attention_bwd_parts")


def lpk_attention_parts(B, S, H, dh, backward):
    return lib().lpk_attention_parts(_i(B), _i(S), _i(H), _i(dh), _i(backward))


# Entry points that serving calls once a token and layer: their argument types are declared once, and plain numbers go in as they are.
_vp, _u32 = C.c_void_p, C.c_uint32
_TYPES = {
    "lpk_linear_attention_fwd": (_i, [_i] + [_vp] * 6 + [_i] * 4 + [_vp, _sz, _vp]),
    "lpk_linear_attention_bwd": (_i, [_i] + [_vp] * 8 + [_i] * 4 + [_vp, _sz, _vp]),
    "lpk_linear_attention_scratch": (_sz, [_i] * 5),
    "lpk_linear_attention_step": (_i, [_i] + [_vp] * 4 + [_i] * 3 + [_vp]),
    "lpk_dropout": (_i, [_i] + [_vp] * 3 + [_sz, _f, _vp, _u32, _vp]),
    "lpk_rmsnorm_fwd": (_i, [_i] + [_vp] * 8 + [_i, _i, _f, _f, _vp, _u32, _vp]),
    "lpk_rmsnorm_bwd": (_i, [_i] + [_vp] * 8 + [_i] * 3 + [_f, _vp, _u32, _vp, _sz, _vp]),
    "lpk_rmsnorm_scratch": (_sz, [_i] * 2),
    "lpk_rotary": (_i, [_i] + [_vp, _i64] * 2 + [_vp] * 2 + [_i] * 6 + [_f, _i, _vp]),
    "lpk_rotary_frequencies": (_i, [_vp, _i] + [C.c_double] * 5),
    "lpk_cache_append": (_i, [_i] + [_vp, _i64] * 2 + [_i] + [_vp] * 7 + [_i] * 7 + [_vp]),
    "lpk_cache_read": (_i, [_i] + [_vp, _i64] * 2 + [_i] + [_vp] * 7 + [_i] * 7 + [_vp]),
    "lpk_cache_attention": (_i, [_i, _vp, _i64, _i] + [_vp] * 8 + [_i64, _vp] + [_i] * 9 + [_vp, _sz, _vp]),
    "lpk_cache_attention_scratch": (_sz, [_i] * 7),
}
_entry = {}


def _fn(name):
    f = _entry.get(name)
    if f is None:
        f = _entry[name] = C.CFUNCTYPE(_TYPES[name][0], *_TYPES[name][1])((name, lib()))
    return f


_T = {}          # element types by the dtype argument, and of the lengths, the 8-bit values and the generator's numbers


def _real(dtype):
    """Types of the operands of a dtype argument; a call's first one fills the table."""
    if not _T:
        import torch
        _T.update({0: (torch.float32,), 1: (torch.bfloat16,), "i32": (torch.int32,), "u64": (torch.int64, torch.uint64),
                   "e4m3": (torch.float8_e4m3fn, torch.uint8), "f64": (torch.float64,), "torch": torch})
    if dtype in (0, 1):
        return _T[dtype]
    raise KernelError(f"dtype {dtype!r}: 0 (fp32) or 1 (bf16) is needed")


def _at(t, types, n, dev):
    """Address of a tensor (None: none) of one of the types (None: nothing reads it) with n elements at least, on the device of that number."""
    if t is None:
        return None
    if (types is None or t.dtype in types) and t.numel() >= n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    raise KernelError(f"{t.dtype} tensor of {tuple(t.shape)}, strides {t.stride()} on {t.device}: at least {n} contiguous elements of "
                      f"{'any type' if types is None else ' or '.join(map(str, types))} on the first tensor's device are needed")


def _none(name):
    raise KernelError(f"{name}: no tensor")


def _run(name, dev, *args):
    """Calls entry point `name`, its last argument the current stream of device number dev."""
    if dev < 0:
        raise KernelError(f"{name}: tensors on the host")
    torch = _T["torch"]
    # the device's number and the stream's handle without the objects around them: 0.2 us instead of 3.3, of 6 for a call
    rt = torch._C
    if dev == rt._cuda_getDevice():
        rc = (_entry.get(name) or _fn(name))(*args, rt._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            rc = _fn(name)(*args, rt._cuda_getCurrentRawStream(dev))
    if rc:
        _ck(rc, name)


def _wide(*n):
    """For numbers that would reach a call cut to 32 bits, when the tensors have been compared with what they were before."""
    raise KernelError(f"{', '.join(map(str, n))}: numbers of 31 bits are needed")


def _size(t):
    return 0 if t is None else t.numel()


def lpk_linear_attention_scratch(B, S, H, dh, backward):
    """Floats of workspace (0 for what the calls refuse); needs no device."""
    return 0 if (B | S | H | dh) >> 31 else _fn("lpk_linear_attention_scratch")(B, S, H, dh, backward)


def lpk_linear_attention_fwd(dtype, qkv, log_decay, lens, s0, o, s_out, B, S, H, dh, scratch=None):
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_linear_attention_fwd") if qkv is None else qkv.get_device()
    if (B | S | H | dh) < 0:
        _wide(B, S, H, dh)
    e = e if S else None
    f, n, state = _T[0], B * S * H * dh, B * H * dh * dh
    _run("lpk_linear_attention_fwd", dev, dtype, _at(qkv, e, 3 * n, dev), _at(log_decay, f, H, dev), _at(lens, _T["i32"], B, dev),
         _at(s0, f, state, dev), _at(o, e, n, dev), _at(s_out, f, state, dev), B, S, H, dh, _at(scratch, f, 0, dev), _size(scratch))


def lpk_linear_attention_bwd(dtype, qkv, log_decay, lens, s0, dout, ds_out, dqkv, ds0, B, S, H, dh, scratch=None):
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_linear_attention_bwd") if qkv is None else qkv.get_device()
    if (B | S | H | dh) < 0:
        _wide(B, S, H, dh)
    e = e if S else None
    f, n, state = _T[0], B * S * H * dh, B * H * dh * dh
    _run("lpk_linear_attention_bwd", dev, dtype, _at(qkv, e, 3 * n, dev), _at(log_decay, f, H, dev), _at(lens, _T["i32"], B, dev),
         _at(s0, f, state, dev), _at(dout, e, n, dev), _at(ds_out, f, state, dev), _at(dqkv, e, 3 * n, dev), _at(ds0, f, state, dev), B, S, H, dh,
         _at(scratch, f, 0, dev), _size(scratch))


def lpk_linear_attention_step(dtype, qkv, log_decay, state, o, B, H, dh):
    e, dev, n = _T.get(dtype) or _real(dtype), _none("lpk_linear_attention_step") if qkv is None else qkv.get_device(), B * H * dh
    if (B | H | dh) < 0:
        _wide(B, H, dh)
    f = _T[0]
    _run("lpk_linear_attention_step", dev, dtype, _at(qkv, e, 3 * n, dev), _at(log_decay, f, H, dev), _at(state, f, n * dh, dev), _at(o, e, n, dev),
         B, H, dh)


def _site(site):
    raise KernelError(f"site {site}: a number of 32 bits is needed")


def lpk_dropout(dtype, x, res, y, p, rng, site):
    """rng: two 64-bit integers (seed, step) on the device."""
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_dropout") if x is None else x.get_device()
    n = x.numel()
    _run("lpk_dropout", dev, dtype, _at(x, e, n, dev), _at(res, e, n, dev), _at(y, e, n, dev), n, p, _at(rng, _T["u64"], 2, dev),
         site if -1 < site < 1 << 32 else _site(site))


def lpk_rmsnorm_scratch(rows, d):
    """Floats of workspace (0 for what the call refuses); needs no device."""
    return 0 if (rows | d) >> 31 else _fn("lpk_rmsnorm_scratch")(rows, d)


def lpk_rmsnorm_fwd(dtype, x, res, g, r, y, y8, y8_scale, rstd, rows, d, eps, p=0.0, rng=None, site=0):
    e, dev, n = _T.get(dtype) or _real(dtype), _none("lpk_rmsnorm_fwd") if x is None else x.get_device(), rows * d
    if (rows | d) < 0:
        _wide(rows, d)
    f = _T[0]
    _run("lpk_rmsnorm_fwd", dev, dtype, _at(x, e, n, dev), _at(res, e, n, dev), _at(g, f, d, dev), _at(r, e, n, dev), _at(y, e, n, dev),
         _at(y8, _T["e4m3"], n, dev), _at(y8_scale, f, rows, dev), _at(rstd, f, rows, dev), rows, d, eps, p, _at(rng, _T["u64"], 2, dev),
         site if -1 < site < 1 << 32 else _site(site))


def lpk_rmsnorm_bwd(dtype, dy, r, rstd, g, add, dres, dx, dg, rows, d, accumulate=0, scratch=None, p=0.0, rng=None, site=0):
    e, dev, n = _T.get(dtype) or _real(dtype), _none("lpk_rmsnorm_bwd") if dy is None else dy.get_device(), rows * d
    if (rows | d) < 0:
        _wide(rows, d)
    f = _T[0]
    _run("lpk_rmsnorm_bwd", dev, dtype, _at(dy, e, n, dev), _at(r, e, n, dev), _at(rstd, f, rows, dev), _at(g, f, d, dev), _at(add, e, n, dev),
         _at(dres, e, n, dev), _at(dx, e, n, dev), _at(dg, f, d, dev), rows, d, accumulate, p, _at(rng, _T["u64"], 2, dev),
         site if -1 < site < 1 << 32 else _site(site), _at(scratch, f, 0, dev), _size(scratch))


def _mat(t, types, rows, cols, dev):
    """Address and leading dimension of a matrix of one of the types with so many rows and columns at least, whose rows are contiguous and do not
    overlap, on the device of that number."""
    if t is None:
        return None, cols
    if t.dtype in types and t.dim() == 2 and t.get_device() == dev:
        (m, n), (ld, one) = t.shape, t.stride()
        if m >= rows and n >= cols and (one == 1 or n == 1) and (ld >= n or m < 2):
            return t.data_ptr(), ld if ld > cols else cols
    raise KernelError(f"{t.dtype} tensor of {tuple(t.shape)}, strides {t.stride()} on {t.device}: a matrix of at least {rows} rows of {cols} contiguous elements of "
                      f"{' or '.join(map(str, types))} on the first tensor's device is needed")


def lpk_rotary_frequencies(rot, base=10000.0, factor=1.0, low=1.0, high=1.0, context=0.0):
    """Host tensor of rot / 2 doubles, radians a position; needs no device."""
    import torch
    if rot >> 31:
        _wide(rot)
    freq = torch.empty(rot // 2, dtype=torch.float64)
    _ck(_fn("lpk_rotary_frequencies")(freq.data_ptr(), rot, base, factor, low, high, context), "lpk_rotary_frequencies")
    return freq


def lpk_rotary(dtype, x, y, pos, freq, rows, S, heads, dh, rot, interleaved=0, scale=1.0, backward=0):
    """x and y: matrices, their rows any distance apart (the q and k columns of qkv, say)."""
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_rotary") if x is None else x.get_device()
    if (rows | S | heads | dh | rot) >> 31:
        _wide(rows, S, heads, dh, rot)
    _run("lpk_rotary", dev, dtype, *_mat(x, e, rows, heads * dh, dev), *_mat(y, e, rows, heads * dh, dev), _at(pos, _T["i32"], rows, dev),
         _at(freq, _T["f64"], rot // 2, dev), rows, S, heads, dh, rot, 1 if interleaved else 0, scale, 1 if backward else 0)


def _pages(table, kpages, B, Hkv, dh, page):
    """Page numbers of a sequence in the table (in one dimension: of B sequences, one behind another), and pages in the pools."""
    n = 0 if kpages is None else kpages.numel() // max(1, Hkv * dh * page)
    if table is None:
        return 0, n
    if table.dim() == 2:
        return table.shape[1], n
    if table.dim() == 1:
        return table.numel() // max(1, B), n
    raise KernelError(f"table of {tuple(table.shape)}: a row of page numbers for each of {B} sequences is needed")


def lpk_cache_append(dtype, k, v, starts, lens, table, kpages, vpages, kscale, vscale, B, T, Hkv, dh, page):
    """k and v: matrices, their rows any distance apart.  The table has a row for each sequence, B or more, as long as it has columns; the pools as many pages as kpages holds."""
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_cache_append") if k is None else k.get_device()
    (most, n), i32, f, q, rows = _pages(table, kpages, B, Hkv, dh, page), _T["i32"], _T[0], _T["e4m3"], k.shape[0]
    if (B | T | Hkv | dh | page | rows | most | n) >> 31:
        _wide(B, T, Hkv, dh, page, rows, most, n)
    _run("lpk_cache_append", dev, dtype, *_mat(k, e, rows, Hkv * dh, dev), *_mat(v, e, rows, Hkv * dh, dev), rows, _at(starts, i32, B + 1, dev),
         _at(lens, i32, B, dev), _at(table, i32, B * most, dev), _at(kpages, q, 0, dev), _at(vpages, q, n * Hkv * dh * page, dev), _at(kscale, f, n * Hkv, dev),
         _at(vscale, f, n * Hkv, dev), B, T, Hkv, dh, page, most, n)


def lpk_cache_read(dtype, k, v, starts, lens, table, kpages, vpages, kscale, vscale, B, T, Hkv, dh, page):
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_cache_read") if k is None else k.get_device()
    (most, n), i32, f, q, rows = _pages(table, kpages, B, Hkv, dh, page), _T["i32"], _T[0], _T["e4m3"], k.shape[0]
    if (B | T | Hkv | dh | page | rows | most | n) >> 31:
        _wide(B, T, Hkv, dh, page, rows, most, n)
    _run("lpk_cache_read", dev, dtype, *_mat(k, e, rows, Hkv * dh, dev), *_mat(v, e, rows, Hkv * dh, dev), rows, _at(starts, i32, B + 1, dev),
         _at(lens, i32, B, dev), _at(table, i32, B * most, dev), _at(kpages, q, 0, dev), _at(vpages, q, n * Hkv * dh * page, dev), _at(kscale, f, n * Hkv, dev),
         _at(vscale, f, n * Hkv, dev), B, T, Hkv, dh, page, most, n)


def lpk_cache_attention_scratch(B, T, H, Hkv, dh, page, max_pages):
    """Floats of workspace (0 for what the call refuses); needs no device."""
    return 0 if (B | T | H | Hkv | dh | page | max_pages) >> 31 else _fn("lpk_cache_attention_scratch")(B, T, H, Hkv, dh, page, max_pages)


def lpk_cache_attention(dtype, q, starts, lens, table, kpages, vpages, kscale, vscale, o, lse, B, T, H, Hkv, dh, page, causal=1, scratch=None):
    """q and o: matrices, their rows any distance apart."""
    e, dev = _T.get(dtype) or _real(dtype), _none("lpk_cache_attention") if q is None else q.get_device()
    (most, n), i32, f, e8, rows = _pages(table, kpages, B, Hkv, dh, page), _T["i32"], _T[0], _T["e4m3"], q.shape[0]
    if (B | T | H | Hkv | dh | page | rows | most | n) >> 31:
        _wide(B, T, H, Hkv, dh, page, rows, most, n)
    _run("lpk_cache_attention", dev, dtype, *_mat(q, e, rows, H * dh, dev), rows, _at(starts, i32, B + 1, dev), _at(lens, i32, B, dev),
         _at(table, i32, B * most, dev), _at(kpages, e8, 0, dev), _at(vpages, e8, n * Hkv * dh * page, dev), _at(kscale, f, n * Hkv, dev),
         _at(vscale, f, n * Hkv, dev), *_mat(o, e, rows, H * dh, dev), _at(lse, f, rows * H, dev), B, T, H, Hkv, dh, page, most, n, 1 if causal else 0,
         _at(scratch, f, 0, dev), _size(scratch))


def lpk_layernorm_fwd(dtype, x, g, b, y, mean, rstd, rows, d):
    _ck(lib().lpk_layernorm_fwd(_i(dtype), _p(x), _p(g), _p(b), _p(y), _p(mean), _p(rstd), _i(rows), _i(d), _stream()),
        "lpk_layernorm_fwd")


def lpk_layernorm_bwd_static(dtype, dy, x, mean, rstd, g, add, dx, dg, db, rows, d, accumulate):
    rc = lib().lpk_layernorm_bwd_static(_i(dtype), _p(dy), _p(x), _p(mean), _p(rstd), _p(g), _p(add), _p(dx), _p(dg),
                                        _p(db), _i(rows), _i(d), _i(accumulate), _stream())
    if rc == 1:
        raise KernelError(f"lpk_layernorm_bwd_static: rows={rows}, d={d} exceed the built-in workspace "
                          f"(((rows + 7) // 8) * d * 2 must be <= {1 << 21})")
    _ck(rc, "lpk_layernorm_bwd_static")


def lpk_layernorm_bwd(dtype, dy, x, mean, rstd, g, add, dx, dg, db, rows, d, accumulate, scratch):
    _ck(lib().lpk_layernorm_bwd(_i(dtype), _p(dy), _p(x), _p(mean), _p(rstd), _p(g), _p(add), _p(dx), _p(dg), _p(db),
                                _i(rows), _i(d), _i(accumulate), _p(scratch), _sz(scratch.numel()), _stream()),
        "lpk_layernorm_bwd")


def lpk_softmax_ce(dtype, z, ld, y, loss_rows, rows, n, write_grad, inv_rows):
    _ck(lib().lpk_softmax_ce(_i(dtype), _p(z), _i64(ld), _p(y), _p(loss_rows), _i(rows), _i(n), _i(write_grad),
                             _f(inv_rows), _stream()), "lpk_softmax_ce")


def lpk_optimizer(kind, lr, momentum, beta1, beta2, eps, weight_decay, t, grad_scale, p, g, m, v, p_bf16, n):
    _ck(lib().lpk_optimizer(_i(kind), _f(lr), _f(momentum), _f(beta1), _f(beta2), _f(eps), _f(weight_decay), _i(t),
                            _f(grad_scale), _p(p), _p(g), _p(m), _p(v), _p(p_bf16), _sz(n), _stream()),
        "lpk_optimizer")


def lpk_copy(src, dst, nbytes):
    _ck(lib().lpk_copy(_p(src), _p(dst), _sz(nbytes), _stream()), "lpk_copy")


def lpk_transpose_bf16(src, dst, R, C):
    _ck(lib().lpk_transpose_bf16(_p(src), _p(dst), _i(R), _i(C), _stream()), "lpk_transpose_bf16")


def lpk_embed_bwd(dtype, ids, dh, demb, T, V, d, accumulate=0, scratch=None):
    _ck(lib().lpk_embed_bwd(_i(dtype), _p(ids), _p(dh), _p(demb), _i(T), _i(V), _i(d), _i(accumulate), _p(scratch),
                            _sz(0 if scratch is None else scratch.numel()), _stream()), "lpk_embed_bwd")


def lpk_conv_fwd(dtype, x, w, out, N, H, W, Cin, O, R, stride, pad):
    _ck(lib().lpk_conv_fwd(_i(dtype), _p(x), _p(w), _p(out), _i(N), _i(H), _i(W), _i(Cin), _i(O), _i(R), _i(stride),
                           _i(pad), _stream()), "lpk_conv_fwd")


def lpk_conv_bwd_data(dtype, dout, w, dx, N, H, W, Cin, O, R, stride, pad):
    _ck(lib().lpk_conv_bwd_data(_i(dtype), _p(dout), _p(w), _p(dx), _i(N), _i(H), _i(W), _i(Cin), _i(O), _i(R),
                                _i(stride), _i(pad), _stream()), "lpk_conv_bwd_data")


def lpk_conv_bwd_weight(dtype, dout, x, dw, N, H, W, Cin, O, R, stride, pad, accumulate=0):
    _ck(lib().lpk_conv_bwd_weight(_i(dtype), _p(dout), _p(x), _p(dw), _i(N), _i(H), _i(W), _i(Cin), _i(O), _i(R),
                                  _i(stride), _i(pad), _i(accumulate), _stream()), "lpk_conv_bwd_weight")


def lpk_conv_bwd_weight_ws(dtype, dout, x, dw, N, H, W, Cin, O, R, stride, pad, splitk_ws, accumulate=0):
    _ck(lib().lpk_conv_bwd_weight_ws(_i(dtype), _p(dout), _p(x), _p(dw), _i(N), _i(H), _i(W), _i(Cin), _i(O), _i(R),
                                     _i(stride), _i(pad), _i(accumulate), _p(splitk_ws), _sz(splitk_ws.numel()),
                                     _stream()), "lpk_conv_bwd_weight_ws")


def lpk_conv_weight_grads(douts, xs, dws, dims, splitk_ws, accumulate=0):
    """dims: (N, H, W, C, O, R, stride, pad) of each convolution."""
    n, vp = len(dws), C.c_void_p * len(dws)
    ptrs = lambda ts: vp(*[t.data_ptr() for t in ts])
    _ck(lib().lpk_conv_weight_grads(_i(n), ptrs(douts), ptrs(xs), ptrs(dws), (C.c_int * (8 * n))(*[v for d in dims for v in d]),
                                    _i(accumulate), _p(splitk_ws), _sz(splitk_ws.numel()), _stream()), "lpk_conv_weight_grads")


def lpk_conv_tile(direction, a, b, out, N, H, W, Cin, O, R, stride, pad, shape, pieces=1, add=None, accumulate=0, stats=None,
                  splitk_ws=None):
    """Returns the rows of a tile whose column sums were left in `stats` (0: none)."""
    rows = C.c_int(0)
    _ck(lib().lpk_conv_tile(_i(direction), _p(a), _p(b), _p(out), _p(add), _i(accumulate), _i(N), _i(H), _i(W), _i(Cin), _i(O),
                            _i(R), _i(stride), _i(pad), _i(shape), _i(pieces), _p(stats),
                            _sz(0 if stats is None else stats.numel()), C.byref(rows), _p(splitk_ws),
                            _sz(0 if splitk_ws is None else splitk_ws.numel()), _stream()), "lpk_conv_tile")
    return rows.value


def lpk_conv_plan(direction, N, H, W, Cin, O, R, stride, pad, splitk_ws_elems):
    """(tile shape, pieces); needs no device."""
    shape, pieces = C.c_int(-1), C.c_int(0)
    _ck(lib().lpk_conv_plan(_i(direction), _i(N), _i(H), _i(W), _i(Cin), _i(O), _i(R), _i(stride), _i(pad), _sz(splitk_ws_elems),
                            C.byref(shape), C.byref(pieces)), "lpk_conv_plan")
    return shape.value, pieces.value


def lpk_conv_bn_fwd(dtype, x, w, z, g, b, res, y, mean, rstd, N, H, W, Cin, O, R, stride, pad, relu, scratch):
    _ck(lib().lpk_conv_bn_fwd(_i(dtype), _p(x), _p(w), _p(z), _p(g), _p(b), _p(res), _p(y), _p(mean), _p(rstd), _i(N),
                              _i(H), _i(W), _i(Cin), _i(O), _i(R), _i(stride), _i(pad), _i(relu), _p(scratch),
                              _sz(scratch.numel()), _stream()), "lpk_conv_bn_fwd")


def lpk_batchnorm_fwd(dtype, z, g, b, res, y, mean, rstd, rows, Cc, relu, scratch):
    _ck(lib().lpk_batchnorm_fwd(_i(dtype), _p(z), _p(g), _p(b), _p(res), _p(y), _p(mean), _p(rstd), _i(rows), _i(Cc),
                                _i(relu), _p(scratch), _sz(scratch.numel()), _stream()), "lpk_batchnorm_fwd")


def lpk_batchnorm_bwd(dtype, dy, y, z, mean, rstd, g, dz, dres, dg, db, rows, Cc, relu, accumulate, scratch):
    _ck(lib().lpk_batchnorm_bwd(_i(dtype), _p(dy), _p(y), _p(z), _p(mean), _p(rstd), _p(g), _p(dz), _p(dres), _p(dg),
                                _p(db), _i(rows), _i(Cc), _i(relu), _i(accumulate), _p(scratch), _sz(scratch.numel()),
                                _stream()), "lpk_batchnorm_bwd")
