"""Calls on pages and draws with nothing to do: no GPU needed, nothing is launched."""
import ctypes as C
import os
import types

import pytest
import torch

from paper_2605_07230_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_07230_amd import build
        build.build(verbose=False)
    return B.load_library()


@pytest.fixture
def ctx(lib):
    """A context made of its limits alone, which nothing but the checks looks at."""
    buf = C.create_string_buffer(4096)
    C.memmove(C.addressof(buf) + 8, C.byref(B.cascade_limits(4, 64, 32, 1000, 8, 128, 256, 4096)), C.sizeof(B.cascade_limits))
    return types.SimpleNamespace(lib=lib, handle=C.addressof(buf), buf=buf)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are the host's")
def test_no_tokens_no_rows(ctx):
    pool = _bf16(2, 10, 2, 16, 64)
    B.paged_append(ctx, k_new=_bf16(2, 0, 2, 64), v_new=_bf16(2, 0, 2, 64), slot_map=_i32(0), k_pages=pool, v_pages=pool)
    B.paged_append(ctx, k_new=_bf16(2, 5, 2, 64), v_new=_bf16(2, 5, 2, 64), slot_map=_i32(0), source=_i32(0), k_pages=pool, v_pages=pool)
    B.paged_append(ctx, k_new=_bf16(0, 5, 2, 64), v_new=_bf16(0, 5, 2, 64), slot_map=_i32(5), k_pages=pool[:0], v_pages=pool[:0])
    for rows, tokens in ((3, 0), (0, 0)):
        q, kv = _bf16(tokens, 8, 64), _bf16(tokens, 2, 64)
        args = dict(q_off=_i32(rows + 1), prefix_len=_i32(rows), block_table=_i32(rows, 4), q=q, k_new=kv, v_new=kv, k_pages=pool[0], v_pages=pool[0],
                    out=torch.empty_like(q), max_new=0, max_prefix_len=0)
        B.paged_attn(ctx, **args)
        assert B.paged_attn_workspace(ctx, **args) == 0
    B.sample_tokens(ctx, logits=torch.zeros(0, 100), u=torch.zeros(0), token=_i32(0), prob=torch.zeros(0))
    B.paged_slots(ctx, seq_len=_i32(0), new_len=_i32(0), block_table=_i32(0, 4), free_pages=_i32(3), free_count=_i32(1), page_size=16, n_pages=10, q_off=_i32(1),
                  slot_map=_i32(0), seq_len_out=_i32(0), free_count_out=_i32(1))


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are the host's")
def test_no_rows_write_nothing(ctx):
    """Host memory stands for the outputs: a kernel, or a copy, would not leave it."""
    out = [torch.full((n,), 77, dtype=torch.int32) for n in (1, 6, 6, 6, 1)]
    for path in (dict(new_len=_i32(0)), dict(node_off=_i32(1), row_prompt=_i32(0), accept_len=_i32(2), path_nodes=_i32(2, 5), n_nodes_total=9)):
        B.paged_slots(ctx, seq_len=_i32(0), block_table=_i32(0, 4), free_pages=_i32(3), free_count=_i32(1), page_size=16, n_pages=10, q_off=out[0], slot_map=out[1],
                      position=out[2], source=out[3], seq_len_out=_i32(0), free_count_out=out[4], **path)
    assert all((x == 77).all() for x in out)


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are the host's")
def test_no_tokens_but_wrong(ctx):
    """What does not depend on the tokens is refused all the same."""
    pool = _bf16(2, 10, 2, 24, 64)
    with pytest.raises(B.CascadeError) as e:
        B.paged_append(ctx, k_new=_bf16(2, 0, 2, 64), v_new=_bf16(2, 0, 2, 64), slot_map=_i32(0), k_pages=pool, v_pages=pool)
    assert e.value.status == B.ESHAPE
    a = B.paged_append_args(B.BF16, 2, 3, 3, 2, 64, None, None, None, None, 64, 64, 20480, 2048, 1024, 64, 10, 16)
    assert ctx.lib.paged_append(ctx.handle, C.byref(a)) == B.EINVAL
