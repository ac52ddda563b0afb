"""Refusals of the calls on pages and draws that the host decides, without a GPU: a context made of its limits alone, which nothing but the checks looks at."""
import ctypes as C
import os

import pytest
import torch

from paper_2605_07230_amd import binding as B

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are made up: tests marked gpu cover refusals on a device")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_07230_amd import build
        build.build(verbose=False)
    return B.load_library()


@pytest.fixture
def ctx():
    buf = C.create_string_buffer(4096)                 # a stream (none), then the limits
    C.memmove(C.addressof(buf) + 8, C.byref(B.cascade_limits(4, 64, 32, 1000, 8, 128, 256, 4096)), C.sizeof(B.cascade_limits))
    return buf


def _refused(fn, ctx, record, changes):
    for status, fields in changes:
        a = type(record).from_buffer_copy(record)
        for k, v in fields.items():
            setattr(a, k, v)
        assert fn(C.addressof(ctx), C.byref(a)) == status, fields


E, S, D = B.EINVAL, B.ESHAPE, B.EDTYPE


def test_null(lib, ctx):
    for name in ("paged_slots", "paged_append", "paged_attn", "sample_tokens"):
        assert getattr(lib, name)(None, None) == E and getattr(lib, name)(C.addressof(ctx), None) == E
    assert lib.paged_attn_workspace(None, None, None) == E


def test_attention(lib, ctx):
    r = B.paged_attn_args(B.BF16, 4, 64, 64, 64, 64, 32, 1000, 8, 2, 128, 0.0, 0, 0, 64, 64, 64, 1024, 256, 64, 64, 4096, 2048, 128, 10, 16, 64, 63, 63, 64, 0, 0, 0)
    _refused(lib.paged_attn, ctx, r, [(E, {k: None}) for k in ("q_off", "prefix_len", "q", "k_new", "v_new", "out", "k_pages", "v_pages", "block_table")]
             + [(E, {k: -1}) for k in ("n_rows", "n_tokens", "max_new", "max_prefix_len", "window", "n_sink", "n_pages", "table_width", "workspace_bytes")]
             + [(E, {k: 72}) for k in ("q", "k_new", "v_new", "k_pages", "v_pages", "out", "workspace")]
             + [(E, dict(scale=float("nan"))), (E, dict(n_pages=0)), (E, dict(table_stride=62)), (E, dict(page_size=0)), (E, dict(n_heads=0)), (D, dict(dtype=2))]
             + [(S, {k: v}) for k, v in (("n_heads", 7), ("n_heads", 9), ("head_dim", 96), ("head_dim", 256), ("page_size", 8), ("page_size", 17), ("page_size", 1040),
                                         ("n_rows", 5), ("n_tokens", 65), ("max_prefix_len", 1001), ("max_new", 33), ("max_new", 0), ("stride_pos", 1 << 26),
                                         ("kv_stride", 1 << 26), ("stride_pos", 129), ("stride_head", -1), ("q_stride", 1016), ("kv_stride", 248), ("n_pages", 1 << 27))])
    _refused(lib.paged_attn, ctx, r, [(S, dict(dtype=B.F32, head_dim=257))])


def test_slots(lib, ctx):
    r = B.paged_slots_args(4, 16, 10, 8, 8, 64, 10, 64, 64, 64, 64, 64, 64, 2, 10, 64, 64, 64, 64, 128, 64, 64, 64, 64, 128)
    _refused(lib.paged_slots, ctx, r, [(E, {k: None}) for k in ("seq_len", "block_table", "free_pages", "free_count", "free_count_out", "q_off", "slot_map", "seq_len_out")]
             + [(E, {k: -1}) for k in ("n_rows", "table_width", "max_tokens", "free_capacity", "n_pages")]
             + [(E, dict(seq_len_out=64)), (E, dict(free_count_out=64)), (E, dict(table_stride=7)), (S, dict(page_size=24)), (S, dict(n_rows=5)),
                (S, dict(n_pages=1 << 28)), (S, dict(table_width=1 << 28, table_stride=1 << 28))]
             + [(E, dict({"new_len": None, k: None})) for k in ("node_off", "row_prompt", "accept_len", "path_nodes", "source")]
             + [(S, dict(new_len=None, max_depth=65)), (S, dict(new_len=None, n_nodes_total=65)), (E, dict(new_len=None, n_prompts=-1)), (B.OK, dict(n_rows=0))])


def test_append(lib, ctx):
    r = B.paged_append_args(B.BF16, 2, 10, 10, 2, 128, 64, 64, 64, 64, 64, 64, 40960, 4096, 2048, 128, 10, 16)
    _refused(lib.paged_append, ctx, r, [(E, {k: None}) for k in ("slot_map", "k_new", "v_new", "k_pages", "v_pages")]
             + [(E, {k: -1}) for k in ("n_layers", "n_tokens", "n_source", "n_kv_heads", "head_dim", "n_pages")]
             + [(E, dict(k_new=72)), (E, dict(source=None, n_source=9)), (D, dict(dtype=5)), (S, dict(head_dim=4)), (S, dict(stride_layer=12)), (S, dict(stride_pos=-8)),
                (S, dict(n_layers=65536)), (S, dict(n_tokens=2 ** 31 - 1)), (S, dict(page_size=40)), (B.OK, dict(n_tokens=0)), (B.OK, dict(n_layers=0))])


def test_draws(lib, ctx):
    r = B.sample_args(B.F32, 3, 4096, 64, 4096, 64, 64, 64, 64, 64, 64, 64)
    _refused(lib.sample_tokens, ctx, r, [(E, {k: None}) for k in ("logits", "u", "token")]
             + [(E, dict(n_rows=-1)), (E, dict(vocab=0)), (D, dict(dtype=2)), (S, dict(vocab=4097)), (S, dict(row_stride=4095)), (B.OK, dict(n_rows=0))])


def test_attention_that_a_launch_cannot_count(lib):
    buf = C.create_string_buffer(4096)
    C.memmove(C.addressof(buf) + 8, C.byref(B.cascade_limits(4, 1 << 30, 32, 1 << 30, 128, 128, 256, 4096)), C.sizeof(B.cascade_limits))
    r = B.paged_attn_args(B.BF16, 4, 64, 0, 64, 1, 1, 1000, 128, 128, 128, 0.0, 0, 0, 64, 64, 64, 16384, 16384, 64, 64, 4096, 2048, 128, 10, 16, 64, 63, 63, 64, 0, 0, 0)
    _refused(lib.paged_attn, buf, r, [(S, dict(n_tokens=(1 << 23) + 1)), (S, dict(dtype=B.F32, n_tokens=(1 << 18) + 1)), (S, dict(max_new=(1 << 30) + 1)),
                                      (S, dict(n_kv_heads=1, max_new=1 << 18)), (B.OK, dict(n_rows=0)), (B.OK, dict(n_tokens=0))])
