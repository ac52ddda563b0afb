"""Tensors with fewer elements than a call on pages reads or writes of them are refused before it, without a GPU: nothing is launched, a stand-in for the library keeps the records."""
from types import SimpleNamespace

import pytest
import torch

from paper_2605_07230_amd import binding as B

S, N, H, KV, D, PAGES, WIDTH, CAP = 3, 7, 4, 2, 64, 5, 2, 40


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


@pytest.fixture
def calls():
    """A context whose library takes every call and keeps its record."""
    kept = []

    class Lib:
        def __getattr__(self, name):
            return lambda handle, record: kept.append((name, record)) or B.OK
    return SimpleNamespace(lib=Lib(), handle=0, kept=kept)


def attention():
    return dict(q_off=i32(S + 1), prefix_len=i32(S), block_table=i32(S, WIDTH), q=bf16(N, H, D), k_new=bf16(N, KV, D), v_new=bf16(N, KV, D), k_pages=bf16(PAGES, KV, 16, D),
                v_pages=bf16(PAGES, KV, 16, D), out=bf16(N, H, D), lse=torch.zeros(N, H), parent=i32(N), max_new=4, max_prefix_len=20)


def shared():
    return dict(attention(), group_off=i32(2), shared_len=i32(1), max_shared_len=16)


def mass():
    return dict(q_off=i32(S + 1), seq_len=i32(S), block_table=i32(S, WIDTH), q=bf16(N, H, D), lse=torch.zeros(N, H), k_pages=bf16(PAGES, KV, 16, D), mass=torch.zeros(S, KV, CAP),
                first=i32(S), prefix_len=i32(S), max_new=4, max_seq_len=20)


def evict():
    return dict(seq_len=i32(S), budget=i32(S), block_table=i32(S, WIDTH), k_pages=bf16(2, PAGES, KV, 16, D), v_pages=bf16(2, PAGES, KV, 16, D), mass=torch.zeros(2, S, KV, CAP),
                mass_out=torch.zeros(2, S, KV, CAP), free_pages=i32(9), free_count=i32(1), seq_len_out=i32(S), free_count_out=i32(1), n_first=i32(S), dropped=i32(S), max_seq_len=20)


BY_ROW = {"paged_attn": (attention, ("q_off", "block_table", "lse", "parent")), "paged_attn_shared": (shared, ("q_off", "block_table", "lse", "parent", "group_off")),
          "paged_mass": (mass, ("q_off", "block_table", "first", "prefix_len")),
          "paged_evict": (evict, ("block_table", "n_first", "seq_len_out", "dropped", "free_count", "free_count_out", "budget"))}


@pytest.mark.parametrize("name", BY_ROW)
def test_short_tensors(name, calls):
    make, names = BY_ROW[name]
    call = getattr(B, name)
    call(calls, **make())
    assert [n for n, _ in calls.kept] == [name + "_record"]
    for k in names:
        args = make()
        args[k] = args[k][:-1]
        with pytest.raises(AssertionError):
            call(calls, **args)
    assert len(calls.kept) == 1


@pytest.mark.parametrize("name", BY_ROW)
def test_longer_buffers_and_what_may_be_missing(name, calls):
    """Buffers made for more rows than a call has are taken, and so is None where the call allows it."""
    make, names = BY_ROW[name]
    for k in names:
        if k in ("budget", "group_off"):
            continue                        # these say how many rows and groups there are
        args = make()
        args[k] = torch.cat([args[k], args[k]])
        getattr(B, name)(calls, **args)
    args = make()
    for k in ("lse", "parent", "first", "prefix_len", "n_first", "dropped"):
        if k in args and not (k == "lse" and name == "paged_mass") and not (k == "prefix_len" and "attn" in name):
            args[k] = None
    getattr(B, name)(calls, **args)
    assert len(calls.kept) == len([k for k in names if k not in ("budget", "group_off")]) + 1
