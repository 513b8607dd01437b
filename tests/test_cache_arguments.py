"""What the wrappers of the 8-bit cache make of their arguments, on the host: an entry point that gets through the checks of its tensors ends at "tensors on
the host", and what it would have been called with is looked at before that."""
import pytest

from test_cache_refusals import B_, K, M_, WRAPPED, refused, tensors  # noqa: F401

CACHE = ("lpk_cache_append", "lpk_cache_read", "lpk_cache_attention")


def passed(K, name, args, monkeypatch):  # noqa: F811
    """Numbers that the entry point would be called with."""
    seen = []
    monkeypatch.setattr(K, "_run", lambda name, dev, *a: seen.extend(a))
    getattr(K, name)(*args.values())
    return seen


@pytest.mark.parametrize("name", CACHE)
def test_a_table_with_more_rows_keeps_its_columns(K, name, monkeypatch):  # noqa: F811
    """A program's table of all its slots, of which the first B are at work: a sequence's pages are a row of it."""
    import torch
    args = tensors(name)
    one = passed(K, name, args, monkeypatch)
    most = len(one) - 1 - one[::-1].index(M_)
    assert one[most - 1] == args["page"] and one[most + 1] == args["kpages"].shape[0]
    wide = passed(K, name, args | dict(table=torch.zeros(7 * B_ + 1, M_, dtype=torch.int32)), monkeypatch)
    assert wide[most] == M_
    flat = passed(K, name, args | dict(table=torch.zeros(B_ * M_, dtype=torch.int32)), monkeypatch)
    assert flat[most] == M_


@pytest.mark.parametrize("name", CACHE)
def test_other_tables_are_refused(K, name):  # noqa: F811
    import torch
    args = tensors(name)
    refused(K, name, args | dict(table=torch.zeros(B_ - 1, M_, dtype=torch.int32)), "contiguous")
    refused(K, name, args | dict(table=torch.zeros(B_ - 1, 5 * M_, dtype=torch.int32)), "contiguous")      # enough numbers, too few rows
    refused(K, name, args | dict(table=torch.zeros(B_, 2 * M_, dtype=torch.int32)[:, :M_]), "contiguous")
    refused(K, name, args | dict(table=torch.zeros(B_, M_, 1, dtype=torch.int32)), "row of page numbers")
    refused(K, name, args | dict(table=torch.zeros((), dtype=torch.int32)), "row of page numbers")
