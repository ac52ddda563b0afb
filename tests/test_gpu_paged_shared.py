"""paged_attn_shared against the oracle: groups of every kind, lengths around tiles and pages, trees, both types; what makes a group share less; refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding

from budget_util import Shared
from serving_util import dev

pytestmark = pytest.mark.gpu

def rows(n, *cycle):
    return [cycle[i % len(cycle)] for i in range(n)]


# calls that take the shared keys once: enough rows and keys that it pays
SHARES = {
    "tokens of one prompt": dict(prefix=rows(16, 1030, 1024, 1100, 1025), new=rows(16, 1), groups=[0, 16], shared=[1024], heads=32, kv_heads=32),
    "grouped heads": dict(prefix=rows(34, 1000, 1090, 1024, 1050, 992), new=rows(34, 1), groups=[0, 34], shared=[992], heads=32, kv_heads=8, page=32),
    "groups, a row by itself": dict(prefix=[*rows(20, 1040, 1100), 50, *rows(13, 1028, 1032)], new=rows(34, 1, 1, 2, 1, 3), groups=[0, 20, 21, 34], shared=[1040, 0, 1024], heads=32,
                                    kv_heads=8),
    "empty groups": dict(prefix=rows(36, 1020, 1030), new=rows(36, 1), groups=[0, 0, 20, 20, 36, 36], shared=[64, 1008, 7, 1010, 9], heads=32, kv_heads=16),
    "not whole tiles": dict(prefix=rows(20, 1021, 1020, 1060), new=rows(20, 2, 1, 1), groups=[0, 20], shared=[1008], heads=16, kv_heads=16),
    "nothing of their own": dict(prefix=rows(20, 1024), new=rows(20, 1), groups=[0, 20], shared=[1024], heads=16, kv_heads=16, page=64),
    "rows without tokens": dict(prefix=rows(20, 1040, 1044, 1050), new=rows(20, 0, 1, 0, 2), groups=[0, 20], shared=[1040], heads=16, kv_heads=16),
    "a group without tokens": dict(prefix=rows(36, 1040, 1044), new=[*rows(18, 0), *rows(18, 1, 2)], groups=[0, 18, 36], shared=[1040, 1040], heads=32, kv_heads=16),
    "a row shorter than what is shared": dict(prefix=[*rows(19, 1040, 1044), 300], new=rows(20, 1), groups=[0, 20], shared=[1040], heads=32, kv_heads=16),
    "long": dict(prefix=rows(8, 8200, 8192, 8300), new=rows(8, 1), groups=[0, 8], shared=[8192], heads=32, kv_heads=8, page=1024),
    "narrow heads": dict(prefix=[*rows(20, 2100, 2050), *rows(20, 1990, 2060)], new=rows(40, 1, 4, 3, 2), groups=[0, 20, 40], shared=[2048, 1984], heads=32, kv_heads=8, head_dim=64),
    "narrow, one kv head": dict(prefix=rows(120, 4100, 4110, 4097), new=rows(120, 1, 2), groups=[0, 120], shared=[4096], heads=8, kv_heads=1, head_dim=64, page=32),
    "many query rows": dict(prefix=rows(64, 600, 580), new=rows(64, 4), groups=[0, 64], shared=[576], heads=32, kv_heads=8),
    "trees": dict(prefix=rows(16, 1040, 1050), new=rows(16, 12, 16, 9), groups=[0, 16], shared=[1040], heads=32, kv_heads=32, tree=4),
    "narrow trees": dict(prefix=rows(32, 1040, 1050), new=rows(32, 7, 8, 1), groups=[0, 10, 32], shared=[1040, 1040], heads=64, kv_heads=32, head_dim=64, tree=3),
    "chunks": dict(prefix=rows(16, 1040, 1050), new=rows(16, 12, 16, 9), groups=[0, 16], shared=[1040], heads=32, kv_heads=32),
    "memory by position": dict(prefix=rows(16, 1040, 1050), new=rows(16, 1, 3), groups=[0, 16], shared=[1040], heads=32, kv_heads=32, order="position"),
    "memory by head": dict(prefix=rows(16, 1040, 1050), new=rows(16, 1, 3), groups=[0, 16], shared=[1040], heads=32, kv_heads=32, order="page_inside"),
    "slices of one projection": dict(prefix=rows(16, 1040, 1050), new=rows(16, 1, 3), groups=[0, 16], shared=[1040], heads=32, kv_heads=32, packed_qkv=True, spare=5),
    "scale, large scores": dict(prefix=rows(16, 1040, 1050), new=rows(16, 1, 3), groups=[0, 16], shared=[1040], heads=32, kv_heads=32, scale=0.5, q_scale=3.0),
    "group of 20": dict(prefix=rows(40, 4110, 4100), new=rows(40, 1, 0), groups=[0, 40], shared=[4096], heads=20, kv_heads=4, page=16),
}
SHARES_F32 = {
    "f32": dict(prefix=rows(16, 540, 512), new=rows(16, 1), groups=[0, 16], shared=[512], heads=8, kv_heads=8, head_dim=64),
    "f32 groups": dict(prefix=rows(40, 540, 600), new=rows(40, 1, 2, 0), groups=[0, 12, 12, 40], shared=[528, 512, 540], heads=4, kv_heads=2, head_dim=64),
    "f32 tree": dict(prefix=rows(20, 540, 512), new=rows(20, 4, 3, 1), groups=[0, 20], shared=[512], heads=4, kv_heads=4, head_dim=64, tree=3),
    "f32 odd head": dict(prefix=rows(20, 540, 512), new=rows(20, 1, 2), groups=[0, 20], shared=[512], heads=4, kv_heads=2, head_dim=70),
    "f32 odd head, tree": dict(prefix=rows(20, 540, 512), new=rows(20, 1, 2), groups=[0, 20], shared=[512], heads=4, kv_heads=2, head_dim=101, tree=2),
    "f32 wide head": dict(prefix=rows(8, 1040, 1029), new=rows(8, 2), groups=[0, 8], shared=[1024], heads=4, kv_heads=4, head_dim=256),
    "f32 wide head, odd, slices": dict(prefix=rows(12, 1040, 1029), new=rows(12, 1, 2), groups=[0, 12], shared=[1024], heads=4, kv_heads=4, head_dim=255, packed_qkv=True, spare=3),
    "f32 head of 100, tree": dict(prefix=rows(12, 1040, 1029), new=rows(12, 2, 3), groups=[0, 12], shared=[1024], heads=4, kv_heads=2, head_dim=100, tree=2),
    "f32 wide head, tree": dict(prefix=rows(12, 1040, 1029), new=rows(12, 2, 3), groups=[0, 12], shared=[1024], heads=4, kv_heads=2, head_dim=200, tree=2),
}
# calls that are paged_attn's
ALONE = {
    "few keys": dict(prefix=[310, 304, 700, 305], new=[1, 1, 1, 1], groups=[0, 4], shared=[304], heads=32, kv_heads=32),
    "less than a tile": dict(prefix=[70, 80], new=[1, 1], groups=[0, 2], shared=[48], heads=4, kv_heads=2),
    "nothing shared": dict(prefix=[70, 80], new=[1, 1], groups=[0, 2], shared=[0], heads=4, kv_heads=2),
    "many tokens": dict(prefix=rows(16, 1040, 1050), new=rows(16, 17, 60), groups=[0, 16], shared=[1040], heads=32, kv_heads=32),
    "large trees": dict(prefix=[400, 350, 410], new=[60, 33, 17], groups=[0, 3], shared=[336], heads=8, kv_heads=8, tree=6),
    "window": dict(prefix=rows(16, 1040, 1050), new=rows(16, 1), groups=[0, 16], shared=[1040], heads=32, kv_heads=32, window=500, n_sink=4),
    "rows by themselves": dict(prefix=[1040, 1050, 900], new=[1, 1, 1], groups=[0, 1, 2, 3], shared=[1040, 64, 64], heads=8, kv_heads=8),
    "f32, few keys": dict(prefix=[270, 300, 256], new=[15, 9, 1], groups=[0, 3], shared=[256], heads=8, kv_heads=8, head_dim=64, dtype="f32"),
}
CASES = {**SHARES, **{k: dict(v, dtype="f32") for k, v in SHARES_F32.items()}, **ALONE}


def make(name, seed=0, **more):
    kw = {**CASES[name], **more}
    return Shared(seed, kw.pop("prefix"), kw.pop("new"), kw.pop("groups"), kw.pop("shared"), **kw)


def some_heads(p):
    return sorted({0, p.kv_heads // 2, p.kv_heads - 1})


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("workspace", [False, True])
def test_against_the_oracle(name, workspace):
    print(f"[paged_attn_shared] {name}: workspace {workspace}", flush=True)
    p = make(name, list(CASES).index(name))
    ctx = p.context()
    more = {}
    if workspace:
        size = binding.paged_attn_shared_workspace(ctx, **p.args, out=p.out)
        more["workspace"] = torch.full((max(size // 4, 4),), float("nan"), device="cuda")
    elif name not in ALONE:
        assert p.cut()[1] > 0
    p.run(ctx, **more)
    assert ctx.device_status() == binding.OK
    p.check(some_heads(p))


@pytest.mark.parametrize("seed", range(16))
def test_random_shapes(seed):
    rng = np.random.default_rng(500 + seed)
    n = int(rng.integers(20, 50))
    groups = [0, *sorted(rng.integers(0, n + 1, int(rng.integers(0, 3))).tolist()), n]
    page = int(rng.choice([16, 32, 48, 64, 256]))
    f32 = seed % 4 == 3
    shared = [int(rng.integers(900, 1500)) // page * page for _ in groups[1:]]
    prefix = [max(0, shared[g] + int(rng.integers(-300 if rng.random() < 0.05 else 0, 200))) for g in range(len(shared)) for _ in range(groups[g], groups[g + 1])]
    kv, group = (2, 2) if f32 else (int(rng.choice([16, 32])), int(rng.choice([1, 2, 4])))
    kw = dict(new=[int(x) for x in rng.integers(0, 3 if f32 else 16 // group + 1, n)], heads=kv * group, kv_heads=kv, head_dim=int(rng.choice([64, 96] if f32 else [64, 128])),
              page=page, order=str(rng.choice(["head", "position", "page_inside"])), dtype="f32" if f32 else "bf16", spare=int(rng.integers(0, 3)))
    if rng.random() < 0.4:
        kw.update(tree=3, new=[max(1, x) for x in kw["new"]])
    kw["new"][0] = max(kw["new"][0], 1)
    print(f"[paged_attn_shared] {prefix} {groups} {shared} {kw}", flush=True)
    p = Shared(seed, prefix, kw.pop("new"), groups, shared, **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check(some_heads(p))


def test_which_calls_share():
    for name in CASES:
        kw = CASES[name]
        n, bf16 = len(kw["prefix"]), kw.get("dtype") != "f32"
        cut = binding.paged_shared_cut(n_rows=n, n_groups=len(kw["shared"]), n_tokens=sum(kw["new"]), max_new=max(kw["new"]), max_prefix_len=max(kw["prefix"]),
                                       max_shared_len=max(0, min(max(kw["shared"]), max(kw["prefix"]))), n_heads=kw["heads"], n_kv_heads=kw["kv_heads"],
                                       head_dim=kw.get("head_dim", 128), tree="tree" in kw, window=kw.get("window", 0), dtype=binding.BF16 if bf16 else binding.F32)
        assert (cut[1] > 0) == (name not in ALONE), (name, cut)
    # both shapes of workgroups, few parts and many
    cuts = [binding.paged_shared_cut(n_rows=r, n_groups=1, n_tokens=r * t, max_new=t, max_prefix_len=4200, max_shared_len=4096, n_heads=32, n_kv_heads=8, head_dim=128)[:2]
            for r, t in ((8, 1), (64, 1), (500, 4))]
    assert {c[0] for c in cuts} == {64, 128} and cuts[0][1] > cuts[1][1] > 1


def small(dtype, seed):
    """Two groups of ten rows with an empty one between them."""
    p = Shared(seed, [*rows(10, 1030, 1040), *rows(10, 1100, 1029)], rows(20, 1, 2), [0, 10, 10, 20], [1024, 0, 1024], heads=32 if dtype == "bf16" else 4,
               kv_heads=32 if dtype == "bf16" else 4, dtype=dtype, head_dim=128 if dtype == "bf16" else 64)
    assert p.cut()[1] > 0
    return p


def test_groups_out_of_order_share_nothing_and_set_the_flag():
    for groups in ([0, 13, 12, 20], [1, 2, 3, 20], [0, 2, 3, 19], [0, 2, 3, 21], [-1, 2, 3, 20], [0, 1 << 30, 3, 20]):
        for dtype in ("bf16", "f32"):
            print(f"[paged_attn_shared] {groups} {dtype}", flush=True)
            p = small(dtype, 3)
            ctx = p.context()
            p.run(ctx, group_off=dev(groups))
            assert ctx.device_status() == binding.ETREE
            p.check(some_heads(p))


def test_a_row_that_cannot_be_computed_leaves_its_group_alone():
    for dtype in ("bf16", "f32"):
        for row, length in ((1, -1), (0, 1 << 20), (12, 1101)):
            print(f"[paged_attn_shared] row {row} of length {length} {dtype}", flush=True)
            p = small(dtype, 4)
            lengths = list(p.prefix)
            lengths[row] = length
            ctx = p.context()
            p.run(ctx, prefix_len=dev(lengths))
            assert ctx.device_status() == binding.ETREE
            lo, hi = p.off[row], p.off[row + 1]
            assert (p.out[lo:hi] == 0).all() and (p.lse[lo:hi] == -float("inf")).all()
            want = small(dtype, 4)
            want.run()
            p.out[lo:hi], p.lse[lo:hi] = want.out[lo:hi], want.lse[lo:hi]
            p.check(some_heads(p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_and_values_behind_what_is_attended_do_not_reach_it(dtype):
    """Infinite values among the shared positions reach all, those among a row's own or its new tokens only that row."""
    for value in (float("inf"), -float("inf")):
        p = small(dtype, 6)
        p.v_pages[p.table[0, 2], 1, 5, 7] = value                  # shared position 37
        p.v_pages[p.table[1, 64], 0, 3, 33] = value                # the second row's own position 1027
        p.v_new[p.off[3] + 1, 0, 5] = value
        p.run()
        p.check([0, 1])


def test_outputs_repeat_and_lse_may_be_missing():
    p = small("bf16", 7)
    ctx = p.context()
    p.run(ctx)
    first = p.out.clone()
    p.run(ctx, lse=None)
    assert torch.equal(first, p.out)
    p.run(ctx, group_off=None, shared_len=None, max_shared_len=0)
    p.check(some_heads(p))


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
