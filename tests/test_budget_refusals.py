"""Refusals of paged_attn_shared, paged_mass and paged_evict that the host decides, and calls with nothing to do, without a GPU: a context made of its limits alone, which nothing
but the checks looks at."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2605_07230_amd import binding as B

from test_abi import HEADER

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses here are made up: tests marked gpu cover refusals on a device")

E, S, D = B.EINVAL, B.ESHAPE, B.EDTYPE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_07230_amd import build
        build.build(verbose=False)
    return B.load_library()


@pytest.fixture
def ctx():
    return _context(4, 64, 32, 1000, 8, 128)


def _context(rows, nodes, tree, prefix, heads, head_dim):
    buf = C.create_string_buffer(4096)                 # a stream (none), then the limits
    C.memmove(C.addressof(buf) + 8, C.byref(B.cascade_limits(rows, nodes, tree, prefix, heads, head_dim, 256, 4096)), C.sizeof(B.cascade_limits))
    return buf


def _refused(fn, ctx, record, changes):
    for status, fields in changes:
        a = type(record).from_buffer_copy(record)
        for k, v in fields.items():
            setattr(a, k, v)
        assert fn(C.addressof(ctx), C.byref(a)) == status, fields


def _attention():
    return (B.BF16, 4, 64, 64, 64, 64, 32, 1000, 8, 2, 128, 0.0, 0, 0, 64, 64, 64, 1024, 256, 64, 64, 4096, 2048, 128, 10, 16, 64, 63, 63, 64, 0, 0, 0)


def test_layout_matches_the_header(tmp_path):
    names = ["paged_shared_args", "paged_mass_args", "paged_evict_args"]
    body = "".join(f'  printf("{n} %zu\\n", sizeof({n}));\n' for n in names)
    at = {"paged_shared_args": ["n_groups", "group_off", "shared_len"], "paged_mass_args": ["n_tokens", "scale", "lse", "mass_cap", "mass_stride_head"],
          "paged_evict_args": ["n_recent", "mass_cap", "k_pages", "free_capacity", "workspace_bytes"]}
    body += "".join(f'  printf("{n}.{f} %zu\\n", offsetof({n}, {f}));\n' for n in names for f in at[n])
    src = tmp_path / "sizes.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{HEADER}"\nint main(void) {{\n{body}  return 0;\n}}\n')
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", str(src), "-o", str(tmp_path / "sizes")])
    out = dict(line.split() for line in subprocess.check_output([str(tmp_path / "sizes")], text=True).splitlines())
    for n in names:
        assert int(out[n]) == C.sizeof(getattr(B, n)), n
        for f in at[n]:
            assert int(out[f"{n}.{f}"]) == getattr(getattr(B, n), f).offset, (n, f)


def test_null(lib, ctx):
    for name in ("paged_attn_shared", "paged_mass", "paged_evict"):
        assert getattr(lib, name)(None, None) == E and getattr(lib, name)(C.addressof(ctx), None) == E
    assert lib.paged_attn_shared_workspace(None, None, None) == E and lib.paged_evict_workspace(None, None, None) == E
    assert lib.cascade_paged_shared(None, None, None, None, None, None) == E


def test_shared(lib, ctx):
    r = B.paged_shared_args(*_attention(), 2, 640, 64, 64)
    changes = ([(E, {k: None}) for k in ("q_off", "prefix_len", "q", "k_new", "v_new", "out", "k_pages", "v_pages", "block_table", "group_off", "shared_len")]
               + [(E, {k: -1}) for k in ("n_rows", "n_tokens", "max_new", "window", "n_groups", "max_shared_len")]
               + [(E, dict(q=72)), (E, dict(workspace=72)), (D, dict(dtype=2)), (S, dict(n_heads=7)), (S, dict(max_prefix_len=1001)), (S, dict(max_prefix_len=639)),
                  (S, dict(page_size=17)), (B.OK, dict(n_rows=0)), (B.OK, dict(n_tokens=0))])
    _refused(lib.paged_attn_shared, ctx, r, changes + [(S, dict(max_new=0))])
    n = C.c_int64()
    _refused(lambda c, a: lib.paged_attn_shared_workspace(c, a, C.byref(n)), ctx, r, changes)


def test_mass(lib, ctx):
    r = B.paged_mass_args(B.BF16, 4, 64, 64, 64, 64, 64, 64, 64, 32, 1000, 8, 2, 128, 0.0, 0, 0, 64, 1024, 64, 64, 4096, 2048, 128, 10, 16, 64, 63, 63, 1000, 64, 2000, 1000)
    _refused(lib.paged_mass, ctx, r, [(E, {k: None}) for k in ("q_off", "seq_len", "q", "lse", "k_pages", "block_table", "mass")]
             + [(E, {k: -1}) for k in ("n_rows", "n_tokens", "n_source", "max_new", "max_seq_len", "window", "n_sink", "mass_cap", "n_pages", "table_width")]
             + [(E, {k: 72}) for k in ("q", "k_pages")]
             + [(E, dict(scale=float("nan"))), (E, dict(scale=-1.0)), (E, dict(n_pages=0)), (E, dict(table_stride=62)), (E, dict(n_heads=0)), (E, dict(source=None, n_source=63)), (E, dict(n_source=0)),
                (D, dict(dtype=2))]
             + [(S, {k: v}) for k, v in (("n_heads", 7), ("n_heads", 16), ("head_dim", 96), ("head_dim", 256), ("page_size", 8), ("page_size", 1040), ("n_rows", 5), ("n_tokens", 65),
                                         ("n_source", 65), ("max_seq_len", 1001), ("max_seq_len", 0), ("max_new", 0), ("stride_pos", 129), ("stride_head", -8), ("q_stride", 1016),
                                         ("mass_stride_row", 999), ("mass_stride_head", 999), ("mass_stride_head", -1), ("max_new", 1 << 28),
                                         ("mass_stride_row", 1000), ("mass_stride_row", 1999), ("mass_stride_head", 2000), ("mass_stride_row", 1 << 62))]   # (sums on each other)
             + [(S, dict(mass_stride_row=1000, mass_stride_head=3999)), (S, dict(mass_stride_row=1000, mass_stride_head=1000))]
             + [(S, dict(dtype=B.F32, head_dim=257)), (B.OK, dict(n_rows=0)), (B.OK, dict(n_tokens=0))])


def test_mass_that_a_launch_cannot_count(lib):
    big = _context(1 << 20, 1 << 30, 32, 1 << 30, 128, 128)
    r = B.paged_mass_args(B.BF16, 1 << 15, 64, 64, None, None, None, 0, 0, 1, 1 << 20, 128, 128, 128, 0.0, 0, 0, 64, 16384, 64, 64, 4096, 2048, 128, 10, 16, 64, 63, 63, 1 << 20, 64,
                          1 << 30, 1 << 20)
    _refused(lib.paged_mass, big, r, [(S, dict(n_tokens=1, n_source=1)), (S, dict(n_tokens=(1 << 23) + 1, n_source=1 << 24, n_rows=1)), (B.OK, dict(n_rows=0))])


def test_evict(lib, ctx):
    r = B.paged_evict_args(B.BF16, 2, 4, 2, 128, 64, 64, 64, 10, 1000, 64, 128, 8000, 2000, 1000, 1000, 10, 16, 63, 64, 128, 40960, 4096, 2048, 128, 64, 63, 10, 64, 64, 128, 128, 256,
                           64, 1 << 30)
    changes = ([(E, {k: None}) for k in ("seq_len", "budget", "mass", "mass_out", "k_pages", "v_pages", "block_table", "free_pages", "free_count", "free_count_out", "seq_len_out")]
               + [(E, {k: -1}) for k in ("n_layers", "n_rows", "n_kv_heads", "head_dim", "n_recent", "max_seq_len", "mass_cap", "free_capacity", "n_pages", "table_width",
                                         "workspace_bytes")]
               + [(E, {k: 72}) for k in ("k_pages", "v_pages", "workspace")]
               + [(E, dict(mass_out=64)), (E, dict(seq_len_out=64)), (E, dict(free_count_out=64)), (E, dict(n_pages=0)), (E, dict(table_stride=62)), (D, dict(dtype=2))]
               + [(S, {k: v}) for k, v in (("n_rows", 5), ("max_seq_len", 1001), ("page_size", 24), ("head_dim", 4), ("stride_layer", 12), ("stride_pos", -8), ("mass_stride_layer", 999),
                                           ("mass_stride_row", 999), ("mass_stride_head", 999), ("mass_stride_head", -1), ("n_layers", 1 << 20), ("n_pages", 1 << 28),
                                           ("mass_stride_layer", 4000), ("mass_stride_row", 1000), ("mass_stride_head", 2000), ("stride_layer", 20480), ("stride_page", 2048),
                                           ("stride_page", 0), ("stride_head", 1024), ("stride_pos", 120))]   # (weights, keys on each other)
               + [(E, {k: v}) for k, v in (("dropped", 64), ("dropped", 128), ("budget", 128), ("n_first", 128), ("n_first", 256), ("v_pages", 64))]
               + [(S, dict(table_width=1 << 28, table_stride=1 << 28)), (B.OK, dict(n_rows=0)), (B.OK, dict(n_layers=0))])
    _refused(lib.paged_evict, ctx, r, changes)
    n = C.c_int64()
    _refused(lambda c, a: lib.paged_evict_workspace(c, a, C.byref(n)), ctx, r, changes)
    assert lib.paged_evict_workspace(C.addressof(ctx), C.byref(r), C.byref(n)) == B.OK and n.value == 0
    long = _context(4, 64, 32, 20000, 8, 128)
    r.max_seq_len = 20000
    assert lib.paged_evict_workspace(C.addressof(long), C.byref(r), C.byref(n)) == B.OK and n.value >= 2 * 4 * 2 * 10000 * 8
    _refused(lib.paged_evict, long, r, [(E, dict(workspace=None)), (S, dict(workspace_bytes=n.value - 1)), (B.OK, dict(n_rows=0))])


def test_cuts():
    ask = dict(n_rows=64, n_groups=1, n_tokens=64, max_new=1, max_prefix_len=4800, max_shared_len=4192, n_heads=32, n_kv_heads=8, head_dim=128)
    assert B.paged_shared_cut(**ask)[1] > 0 and B.paged_shared_cut(**{**ask, 'dtype': B.F32})[1] > 0
    for alone in (dict(max_new=5), dict(n_rows=2), dict(max_prefix_len=20000), dict(window=100), dict(n_groups=0), dict(n_groups=64), dict(max_shared_len=63)):
        assert B.paged_shared_cut(**{**ask, **alone})[:2] == (0, 0), alone
    with pytest.raises(B.CascadeError):
        B.paged_shared_cut(**{**ask, "n_rows": 0})
