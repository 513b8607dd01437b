"""Sizes that are the right ones but for a multiple of 2^32, on the host: the wrappers compare tensors with them as they are, the entry points would get them cut to 32
bits, so that what is too small would be taken as large enough."""
import pytest

import test_cache_refusals as cache
import test_residual_refusals as residual
from test_cache_refusals import K  # noqa: F401

OFF = (-(1 << 32), 1 << 32, -(1 << 31), 1 << 31, -(1 << 40))


def numbers(wrapped, names):
    return [(n, a) for n in wrapped for a in names if a in wrapped[n]]


@pytest.mark.parametrize("name,arg", numbers(cache.WRAPPED, ("rows", "S", "heads", "rot", "B", "T", "H", "Hkv", "dh", "page")))
@pytest.mark.parametrize("off", OFF)
def test_cache_and_rotary(K, name, arg, off, monkeypatch):  # noqa: F811
    args = cache.tensors(name)
    calls = []
    monkeypatch.setattr(K, "_run", lambda *a: calls.append(a))
    with pytest.raises(K.KernelError, match="31 bits"):
        getattr(K, name)(*(args | {arg: args[arg] + off}).values())
    assert not calls


@pytest.mark.parametrize("off", OFF)
def test_host_functions(K, off):  # noqa: F811
    with pytest.raises(K.KernelError):
        K.lpk_rotary_frequencies(8 + off)
    size = dict(B=1, T=1, H=8, Hkv=8, dh=64, page=64, max_pages=1000)
    for arg in size:
        assert K.lpk_cache_attention_scratch(*(size | {arg: size[arg] + off}).values()) == 0


@pytest.mark.parametrize("name,arg", numbers(residual.WRAPPED, ("rows", "d", "B", "S", "H", "dh")))
@pytest.mark.parametrize("off", OFF)
def test_residual_chain(K, name, arg, off, monkeypatch):  # noqa: F811
    args = residual.tensors(residual.WRAPPED[name])
    calls = []
    monkeypatch.setattr(K, "_run", lambda *a: calls.append(a))
    with pytest.raises(K.KernelError, match="31 bits" if off < 0 else "at least"):
        getattr(K, name)(*(args | {arg: args[arg] + off}).values())
    assert not calls


@pytest.mark.parametrize("off", OFF)
def test_workspaces_of_the_residual_chain(K, off):  # noqa: F811
    for arg in range(4):
        size = [1, 4096, 2, 64, 0]
        size[arg] += off
        assert K.lpk_linear_attention_scratch(*size) == 0
    assert K.lpk_rmsnorm_scratch(5 + off, 64) == K.lpk_rmsnorm_scratch(5, 64 + off) == 0
