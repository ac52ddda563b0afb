"""paged_attn_shared against the oracle: groups of every kind, lengths around tiles and pages, trees, both types; what makes a group share less; refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding

from budget_util import Shared
from serving_util import dev

pytestmark = pytest.mark.gpu

CASES = {
    "tokens of one prompt": dict(prefix=[310, 304, 700, 305], new=[1, 1, 1, 1], groups=[0, 4], shared=[304], heads=32, kv_heads=32),
    "grouped heads": dict(prefix=[1000, 1090, 1024, 1300, 999, 1500], new=[1] * 6, groups=[0, 6], shared=[992], heads=16, kv_heads=2, page=32),
    "two groups, a row by itself": dict(prefix=[640, 700, 900, 50, 128, 300, 200], new=[1, 1, 2, 1, 3, 1, 1], groups=[0, 3, 4, 7], shared=[640, 0, 128], heads=8, kv_heads=2),
    "empty groups": dict(prefix=[320, 350, 90], new=[1, 1, 1], groups=[0, 0, 2, 2, 3, 3], shared=[64, 320, 7, 64, 9], heads=8, kv_heads=4),
    "not whole tiles": dict(prefix=[200, 201, 190], new=[2, 1, 1], groups=[0, 3], shared=[176], heads=4, kv_heads=4),
    "one tile": dict(prefix=[64, 64], new=[1, 1], groups=[0, 2], shared=[64], heads=4, kv_heads=2),
    "less than a tile": dict(prefix=[70, 80], new=[1, 1], groups=[0, 2], shared=[48], heads=4, kv_heads=2),
    "nothing of their own": dict(prefix=[512, 512, 512], new=[1, 1, 1], groups=[0, 3], shared=[512], heads=8, kv_heads=8, page=64),
    "rows without tokens": dict(prefix=[300, 310, 320, 500], new=[0, 1, 0, 2], groups=[0, 4], shared=[288], heads=4, kv_heads=2),
    "a group without tokens": dict(prefix=[300, 310, 320, 500], new=[0, 0, 1, 2], groups=[0, 2, 4], shared=[288, 320], heads=4, kv_heads=2),
    "a row shorter than what is shared": dict(prefix=[500, 130, 600], new=[1, 1, 1], groups=[0, 3], shared=[448], heads=4, kv_heads=2),
    "long": dict(prefix=[9000, 9100, 8999, 9500], new=[1, 1, 1, 1], groups=[0, 4], shared=[8960], heads=8, kv_heads=2, page=64),
    "narrow heads": dict(prefix=[1500, 1030, 1100, 2000, 90, 95], new=[1, 4, 3, 1, 1, 1], groups=[0, 4, 6], shared=[1024, 80], heads=16, kv_heads=4, head_dim=64),
    "narrow, many": dict(prefix=[700 + 3 * i for i in range(40)], new=[1 + i % 3 for i in range(40)], groups=[0, 40], shared=[704], heads=8, kv_heads=1, head_dim=64, page=32),
    "trees": dict(prefix=[400, 350, 410], new=[60, 33, 17], groups=[0, 3], shared=[336], heads=8, kv_heads=8, tree=6),
    "small trees": dict(prefix=[400, 350, 410, 399], new=[12, 9, 5, 1], groups=[0, 2, 4], shared=[336, 384], heads=4, kv_heads=4, tree=4),
    "chunks": dict(prefix=[300, 256, 400], new=[70, 130, 9], groups=[0, 3], shared=[256], heads=8, kv_heads=2),
    "memory by position": dict(prefix=[330, 259], new=[1, 3], groups=[0, 2], shared=[256], heads=8, kv_heads=4, order="position"),
    "slices of one projection": dict(prefix=[330, 259], new=[1, 3], groups=[0, 2], shared=[256], heads=8, kv_heads=4, packed_qkv=True, spare=5),
    "window": dict(prefix=[400, 390], new=[1, 1], groups=[0, 2], shared=[384], heads=8, kv_heads=2, window=500, n_sink=4),
    "scale, large scores": dict(prefix=[312, 310], new=[3, 4], groups=[0, 2], shared=[304], scale=0.5, q_scale=3.0),
    "large pages": dict(prefix=[1500, 2100], new=[1, 1], groups=[0, 2], shared=[1024], heads=4, kv_heads=2, page=1024),
}
F32 = {
    "f32": dict(prefix=[270, 300, 256], new=[15, 9, 1], groups=[0, 3], shared=[256], heads=8, kv_heads=8, head_dim=64),
    "f32 tree": dict(prefix=[270, 300, 256], new=[15, 9, 30], groups=[0, 3], shared=[256], heads=8, kv_heads=8, head_dim=64, tree=5),
    "f32 odd head": dict(prefix=[270, 300, 256, 90, 100], new=[3, 1, 2, 1, 1], groups=[0, 3, 5], shared=[240, 80], heads=4, kv_heads=2, head_dim=70),
    "f32 wide head": dict(prefix=[330, 400], new=[3, 20], groups=[0, 2], shared=[320], heads=4, kv_heads=4, head_dim=256),
    "f32 head of 100": dict(prefix=[330, 400], new=[3, 20], groups=[0, 2], shared=[320], heads=4, kv_heads=2, head_dim=100, tree=3),
}
ALONE = ("window", "less than a tile")          # calls that are paged_attn's


@pytest.mark.parametrize("name", [*CASES, *F32])
@pytest.mark.parametrize("workspace", [False, True])
def test_against_the_oracle(name, workspace):
    kw = dict(CASES.get(name) or dict(F32[name], dtype="f32"))
    print(f"[paged_attn_shared] {name}: {kw} workspace {workspace}", flush=True)
    p = Shared(list([*CASES, *F32]).index(name), kw.pop("prefix"), kw.pop("new"), kw.pop("groups"), kw.pop("shared"), **kw)
    ctx = p.context()
    more = {}
    if workspace:
        size = binding.paged_attn_shared_workspace(ctx, **p.args, out=p.out)
        more["workspace"] = torch.full((max(size // 4, 4),), float("nan"), device="cuda")
    p.run(ctx, **more)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.default_rng(500 + seed)
    rows = int(rng.integers(2, 20))
    groups = [0, *sorted(rng.integers(0, rows + 1, int(rng.integers(0, 4))).tolist()), rows]
    page = int(rng.choice([16, 32, 48, 64, 256]))
    most = int(rng.choice([100, 400, 1500]))
    shared = [int(rng.integers(0, most)) // page * page for _ in groups[1:]]
    prefix = [max(0, shared[g] + int(rng.integers(-20 if rng.random() < 0.1 else 0, 300))) for g in range(len(shared)) for _ in range(groups[g], groups[g + 1])]
    kv = int(rng.choice([1, 2, 4]))
    kw = dict(new=[int(x) for x in rng.integers(0, rng.choice([2, 5, 40]), rows)], heads=kv * int(rng.choice([1, 2, 4, 5])), kv_heads=kv, head_dim=int(rng.choice([64, 128])),
              page=page, order=str(rng.choice(["head", "position", "page_inside"])), dtype="f32" if seed % 5 == 4 else "bf16", spare=int(rng.integers(0, 3)))
    if max(kw["new"]) == 0:
        kw["new"][0] = 1
    if rng.random() < 0.4:
        kw.update(tree=5, new=[max(1, n) for n in kw["new"]])
    print(f"[paged_attn_shared] {prefix} {groups} {shared} {kw}", flush=True)
    p = Shared(seed, prefix, kw.pop("new"), groups, shared, **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


def test_which_calls_share():
    for name, kw in {**CASES, **{k: dict(v, dtype="f32") for k, v in F32.items()}}.items():
        kw = dict(kw)
        p = Shared(0, kw.pop("prefix"), kw.pop("new"), kw.pop("groups"), kw.pop("shared"), **kw)
        if name in ALONE:
            assert p.cut()[:2] == (0, 0), name
    assert binding.paged_shared_cut(n_rows=64, n_groups=1, n_tokens=64, max_new=1, max_prefix_len=4700, max_shared_len=4192, n_heads=32, n_kv_heads=8, head_dim=128)[1] > 0


def test_groups_out_of_order_share_nothing_and_set_the_flag():
    for groups in ([0, 3, 2, 4], [1, 2, 3, 4], [0, 2, 3, 3], [0, 2, 3, 5], [-1, 2, 3, 4], [0, 1 << 30, 3, 4]):
        for dtype in ("bf16", "f32"):
            print(f"[paged_attn_shared] {groups} {dtype}", flush=True)
            p = Shared(3, [300, 310, 700, 720], [1, 2, 1, 1], [0, 2, 2, 4], [256, 0, 640], heads=4, kv_heads=2, dtype=dtype)
            ctx = p.context()
            p.run(ctx, group_off=dev(groups))
            assert ctx.device_status() == binding.ETREE
            p.check()


def test_a_row_that_cannot_be_computed_leaves_its_group_alone():
    for dtype in ("bf16", "f32"):
        for row, length in ((1, -1), (0, 1 << 20), (2, 1001)):
            print(f"[paged_attn_shared] row {row} of length {length} {dtype}", flush=True)
            p = Shared(4, [300, 310, 320, 900, 1000], [1, 2, 1, 1, 1], [0, 3, 5], [256, 640], heads=4, kv_heads=2, dtype=dtype)
            lengths = list(p.prefix)
            lengths[row] = length
            ctx = p.context()
            p.run(ctx, prefix_len=dev(lengths))
            assert ctx.device_status() == binding.ETREE
            lo, hi = p.off[row], p.off[row + 1]
            assert (p.out[lo:hi] == 0).all() and (p.lse[lo:hi] == -float("inf")).all()
            want = Shared(4, p.prefix, p.new, p.groups, p.shared, heads=4, kv_heads=2, dtype=dtype)
            want.run()
            p.out[lo:hi], p.lse[lo:hi] = want.out[lo:hi], want.lse[lo:hi]
            p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_and_values_behind_what_is_attended_do_not_reach_it(dtype):
    """Infinite values among the shared positions reach all, those among a row's own or its new tokens only that row."""
    for value in (float("inf"), -float("inf")):
        p = Shared(6, [300, 310, 330], [2, 1, 3], [0, 3], [256], heads=4, kv_heads=2, dtype=dtype)
        p.v_pages[p.table[0, 2], 1, 5, 7] = value                  # shared position 37
        p.v_pages[p.table[1, 18], 0, 3, 64] = value                # the second row's own position 291
        p.v_new[p.off[2] + 1, 0, 5] = value
        p.run()
        p.check()


def test_outputs_repeat_and_lse_may_be_missing():
    p = Shared(7, [700, 720, 1000], [1, 5, 2], [0, 3], [640], heads=8, kv_heads=2)
    ctx = p.context()
    p.run(ctx)
    first = p.out.clone()
    p.run(ctx, lse=None)
    assert torch.equal(first, p.out)
    p.run(ctx, group_off=None, shared_len=None, max_shared_len=0)
    p.check()


def test_refusals():
    p = Shared(8, [300, 310], [3, 2], [0, 2], [256], heads=4, kv_heads=2)
    ctx = p.context()
    rec = binding._paged_shared_record(**p.args, out=p.out, lse=p.lse, workspace=None)

    def call(**fields):
        a = binding.paged_shared_args.from_buffer_copy(rec)
        for k, v in fields.items():
            setattr(a, k, v)
        n = C.c_int64()
        st = ctx.lib.paged_attn_shared(ctx.handle, C.byref(a))
        assert ctx.lib.paged_attn_shared_workspace(ctx.handle, C.byref(a), C.byref(n)) == st or fields.get("max_new") == 0
        return st

    E = binding
    for k in ("q_off", "prefix_len", "q", "k_new", "v_new", "out", "k_pages", "v_pages", "block_table", "group_off", "shared_len"):
        assert call(**{k: None}) == E.EINVAL, k
    for k in ("n_rows", "n_tokens", "max_new", "max_prefix_len", "window", "n_groups", "max_shared_len"):
        assert call(**{k: -1}) == E.EINVAL, k
    assert call(dtype=2) == E.EDTYPE
    for k, v in (("page_size", 24), ("n_heads", 5), ("head_dim", 96), ("n_rows", 3), ("max_prefix_len", 311), ("max_new", 0), ("max_shared_len", 311)):
        assert call(**{k: v}) == E.ESHAPE, (k, v)
    assert call(n_rows=0) == E.OK and call(n_tokens=0) == E.OK
    torch.cuda.synchronize()
    assert (p.out == 7).all() and ctx.device_status() == E.OK
