"""paged_attn against the oracle: lengths, page sizes, orders of memory, windows, trees, both types."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding

from serving_util import Problem, dev

pytestmark = pytest.mark.gpu

CASES = {
    "one token, nothing cached": dict(prefix=[0], new=[1]),
    "one token": dict(prefix=[312, 312], new=[1, 1], heads=32, kv_heads=32),
    "lengths around tiles and pages": dict(prefix=[0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200], new=[1] * 12, heads=4, kv_heads=2),
    "few tokens, grouped": dict(prefix=[700, 3, 0, 64], new=[3, 17, 2, 1], heads=16, kv_heads=2),
    "one kv head of 8": dict(prefix=[1000, 90], new=[1, 1], heads=8, kv_heads=1, page=32),
    "group of 3": dict(prefix=[500, 77, 0], new=[1, 9, 33], heads=12, kv_heads=4, page=48),
    "group of 16": dict(prefix=[500, 77, 0], new=[1, 2, 5], heads=16, kv_heads=1),
    "group of 20": dict(prefix=[500, 77, 0], new=[1, 2, 5], heads=20, kv_heads=1),
    "rows without tokens": dict(prefix=[50, 60, 0, 70], new=[0, 5, 0, 1]),
    "long, one row": dict(prefix=[9000], new=[1], heads=4, kv_heads=1, page=64),
    "chunk": dict(prefix=[300], new=[257], heads=8, kv_heads=2),
    "chunks of ragged rows": dict(prefix=[0, 130, 1000, 64], new=[200, 64, 65, 1], heads=4, kv_heads=4, page=128),
    "prompt": dict(prefix=[0], new=[1000], heads=2, kv_heads=1, page=1024),
    "chunk between tokens": dict(prefix=[900, 20, 333, 1200], new=[1, 300, 1, 1], heads=8, kv_heads=2, page=80),
    "narrow heads": dict(prefix=[100, 700, 65], new=[130, 1, 64], heads=8, kv_heads=2, head_dim=64),
    "narrow tokens": dict(prefix=[100, 700, 65, 2100], new=[1, 1, 1, 1], heads=8, kv_heads=8, head_dim=64, page=32),
    "memory by position": dict(prefix=[100, 259], new=[70, 1], heads=8, kv_heads=4, order="position"),
    "memory by head": dict(prefix=[100, 259], new=[70, 1], heads=8, kv_heads=4, order="page_inside"),
    "slices of one projection": dict(prefix=[100, 259], new=[70, 1], heads=8, kv_heads=4, packed_qkv=True, spare=5),
    "window": dict(prefix=[400, 90, 1000], new=[1, 1, 1], heads=8, kv_heads=2, window=100, n_sink=4),
    "window of one": dict(prefix=[400, 0], new=[5, 3], window=1),
    "window, chunk": dict(prefix=[700, 0, 40], new=[300, 333, 1], heads=4, kv_heads=2, window=64, n_sink=3),
    "window that reaches no cached key": dict(prefix=[100, 65], new=[400, 130], heads=4, kv_heads=2, window=50),
    "window, sinks in the chunk": dict(prefix=[5, 0], new=[200, 300], heads=4, kv_heads=2, window=40, n_sink=70),
    "window wider than all": dict(prefix=[100, 7], new=[50, 1], window=5000, n_sink=1),
    "window, many sinks": dict(prefix=[900], new=[100], heads=2, kv_heads=1, window=130, n_sink=200, head_dim=64),
    "window, long": dict(prefix=[6000], new=[40], heads=4, kv_heads=1, window=700, n_sink=1, page=32),
    "trees": dict(prefix=[312, 100, 0], new=[60, 33, 17], heads=8, kv_heads=8, tree=6),
    "tree of one": dict(prefix=[312, 0], new=[1, 1], tree=3),
    "large trees": dict(prefix=[500, 1100], new=[256, 200], heads=8, kv_heads=2, tree=10, page=64),
    "trees, window": dict(prefix=[312, 3, 0], new=[60, 33, 90], heads=4, kv_heads=2, tree=9, window=5, n_sink=6),
    "deep tree": dict(prefix=[70], new=[150], heads=2, kv_heads=2, tree=60, head_dim=64),
    "trees, wide window": dict(prefix=[900, 80], new=[60, 100], heads=4, kv_heads=2, tree=9, window=200, n_sink=1),
    "scale": dict(prefix=[312, 10], new=[3, 40], scale=0.5),
    "large scores": dict(prefix=[312, 10], new=[3, 40], q_scale=12.0),
}
F32 = {
    "f32 one": dict(prefix=[256], new=[15], heads=8, kv_heads=8, head_dim=64),
    "f32 odd head": dict(prefix=[100, 0, 17], new=[3, 20, 1], heads=4, kv_heads=2, head_dim=70),
    "f32 wide head": dict(prefix=[100, 33], new=[30, 1], heads=4, kv_heads=4, head_dim=256),
    "f32 head of 3": dict(prefix=[40], new=[5], heads=2, kv_heads=1, head_dim=3),
    "f32 tree": dict(prefix=[100, 60], new=[60, 130], heads=4, kv_heads=2, head_dim=64, tree=8),
    "f32 window": dict(prefix=[300, 20, 0], new=[100, 1, 90], heads=4, kv_heads=2, head_dim=80, window=30, n_sink=3),
    "f32 long": dict(prefix=[5000, 1], new=[1, 2], heads=4, kv_heads=1, head_dim=128, page=64),
    "f32 slices": dict(prefix=[100, 33], new=[30, 1], heads=4, kv_heads=4, head_dim=72, packed_qkv=True, order="position", spare=2),
    "f32 tree, window": dict(prefix=[100, 3], new=[60, 33], heads=4, kv_heads=2, head_dim=64, tree=8, window=4, n_sink=5),
}


@pytest.mark.parametrize("name", [*CASES, *F32])
def test_against_the_oracle(name):
    kw = dict(CASES.get(name) or dict(F32[name], dtype="f32"))
    print(f"[paged_attn] {name}: {kw}", flush=True)
    p = Problem(list([*CASES, *F32]).index(name), kw.pop("prefix"), kw.pop("new"), **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    rows = int(rng.integers(1, 9))
    tree = int(rng.choice([0, 0, 6]))
    kv = int(rng.choice([1, 2, 4]))
    kw = dict(prefix=[int(x) for x in rng.integers(0, rng.choice([20, 300, 1500]), rows)], new=[int(x) for x in rng.integers(1, rng.choice([2, 20, 300]), rows)],
              heads=kv * int(rng.choice([1, 2, 4, 5])), kv_heads=kv, head_dim=int(rng.choice([64, 128])), page=int(rng.choice([16, 32, 48, 64, 256])),
              order=str(rng.choice(["head", "position", "page_inside"])), tree=tree, dtype="f32" if seed % 6 == 5 else "bf16", spare=int(rng.integers(0, 3)))
    if rng.random() < 0.4:
        kw.update(window=int(rng.integers(1, 400)), n_sink=int(rng.integers(0, 90)))
    print(f"[paged_attn] {kw}", flush=True)
    p = Problem(seed, kw.pop("prefix"), kw.pop("new"), **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_a_token_does_not_attend_do_not_reach_it(dtype, value):
    """Such a key or value in one new token of each row: those that attend it show it, the others are exact."""
    print(f"[paged_attn] masked {value} {dtype}", flush=True)
    for kw in (dict(new=[70, 9], prefix=[100, 0]), dict(new=[70, 40], prefix=[100, 0], tree=6), dict(new=[100, 9], prefix=[100, 30], window=20, n_sink=2)):
        p = Problem(5, heads=4, kv_heads=2, dtype=dtype, **kw)
        p.v_new[30, 0, 5] = value
        p.v_new[30, 1, 64] = value
        p.run()
        p.check()
        p = Problem(6, heads=4, kv_heads=2, dtype=dtype, **kw)
        p.k_new[30] = float("nan")          # (an infinite key gives infinite scores of either sign)
        p.run()
        p.check()


def test_lse_may_be_missing_and_outputs_repeat():
    p = Problem(7, [700, 20], [5, 200], heads=8, kv_heads=2)
    ctx = p.context()
    p.run(ctx)
    first = p.out.clone()
    p.run(ctx, lse=None)
    assert torch.equal(first, p.out)


def test_rows_that_break_their_bounds_get_zeros_and_the_flag():
    for change in (dict(prefix_len=[-1, 50]), dict(prefix_len=[41, 50]), dict(max_new=2), dict(q_off=[0, -4, 6]), dict(q_off=[0, 90, 6]), dict(q_off=[2, 1, 6]),
                   dict(block_width=2)):
        for dtype in ("bf16", "f32"):
            print(f"[paged_attn] {change} {dtype}", flush=True)
            p = Problem(8, [40, 50], [3, 2], heads=4, kv_heads=2, dtype=dtype, spare=1)
            more = dict(max_prefix_len=50)
            if "block_width" in change:                      # tables of 32 positions, prefixes of 40 and 50
                more["block_table"] = p.block_table[:, :2]
            elif "max_new" in change:
                more["max_new"] = 2
            else:
                key, val = next(iter(change.items()))
                if key == "prefix_len" and val[0] == 41:
                    more["max_prefix_len"] = 49              # the second row's prefix is longer than the bound
                    val = [40, 50]
                more[key] = dev(val)
            ctx = p.context()
            p.run(ctx, **more)
            assert ctx.device_status() == binding.ETREE
            assert torch.isfinite(p.out).all()
            bad = {"prefix_len": [0] if change.get("prefix_len") == [-1, 50] else [1], "max_new": [0], "block_width": [0, 1]}.get(next(iter(change)))
            for s in bad or []:
                assert (p.out[p.off[s]:p.off[s + 1]] == 0).all() and (p.lse[p.off[s]:p.off[s + 1]] == -float("inf")).all()
            assert ctx.device_status() == binding.OK


def test_an_entry_outside_the_pool_sets_the_flag():
    for entry in (-1, 1 << 30, -(1 << 31)):
        for dtype in ("bf16", "f32"):
            p = Problem(9, [40, 50], [3, 2], heads=4, kv_heads=2, dtype=dtype)
            p.k_pages.nan_to_num_(0.0)
            p.v_pages.nan_to_num_(0.0)
            table = p.block_table.clone()
            table[0, 1] = entry
            ctx = p.context()
            p.run(ctx, block_table=table)
            assert ctx.device_status() == binding.ETREE
            p.prefix, p.new = [0, 50], [0, 2]                # the row of the good entries
            off = p.off
            p.off = np.array([off[1], off[1], off[2]])
            p.check()


def test_a_parent_behind_its_node_sets_the_flag():
    p = Problem(10, [40], [20], heads=4, kv_heads=2, tree=5)
    parent = p.args["parent"].clone()
    parent[7] = 9
    ctx = p.context()
    p.run(ctx, parent=parent)
    assert ctx.device_status() == binding.ETREE


def test_refusals():
    p = Problem(11, [40, 50], [3, 2], heads=4, kv_heads=2)
    ctx = p.context()
    names = ("q_off", "prefix_len", "block_table", "q", "k_new", "v_new", "k_pages", "v_pages", "parent", "scale", "window", "n_sink", "max_new", "max_prefix_len")
    rec = binding._paged_attn_record(**{k: p.args[k] for k in names}, out=p.out, lse=p.lse, workspace=None)

    def call(**fields):
        a = binding.paged_attn_args.from_buffer_copy(rec)
        for k, v in fields.items():
            setattr(a, k, v)
        n = C.c_int64()
        st = ctx.lib.paged_attn(ctx.handle, C.byref(a))
        assert ctx.lib.paged_attn_workspace(ctx.handle, C.byref(a), C.byref(n)) == st or fields.get("max_new") == 0
        return st

    E = binding
    for k in ("q_off", "prefix_len", "q", "k_new", "v_new", "out", "k_pages", "v_pages", "block_table"):
        assert call(**{k: None}) == E.EINVAL, k
    for k in ("n_rows", "n_tokens", "max_new", "max_prefix_len", "window", "n_sink", "workspace_bytes", "table_width", "n_pages"):
        assert call(**{k: -1}) == E.EINVAL, k
    assert call(dtype=2) == E.EDTYPE
    assert call(scale=float("nan")) == E.EINVAL and call(scale=-1.0) == E.EINVAL
    for k, v in (("page_size", 24), ("page_size", 2048), ("n_heads", 5), ("n_heads", 8), ("head_dim", 96), ("head_dim", 32), ("stride_pos", 4), ("stride_page", 12),
                 ("stride_head", -8), ("q_stride", 8), ("kv_stride", 257), ("n_rows", 3), ("n_tokens", 6), ("max_prefix_len", 51), ("max_new", 0), ("n_pages", 1 << 28)):
        assert call(**{k: v}) == E.ESHAPE, (k, v)
    for k in ("q", "k_new", "v_new", "k_pages", "v_pages", "out", "workspace"):
        a = binding.paged_attn_args.from_buffer_copy(rec)
        assert call(**{k: (getattr(a, k) or 4096) + 8}) == E.EINVAL, k
    assert call(n_rows=0) == E.OK and call(n_tokens=0) == E.OK
    torch.cuda.synchronize()
    assert (p.out == 7).all() and ctx.device_status() == E.OK


def test_no_cache_at_all():
    p = Problem(12, [0, 0], [30, 1], heads=4, kv_heads=2)
    p.run(k_pages=None, v_pages=None, block_table=None)
    p.check()
