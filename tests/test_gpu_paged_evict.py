"""paged_evict against the oracle, bit for bit: every place of the pool and of the lists."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding

from budget_util import Evict
from serving_util import dev

pytestmark = pytest.mark.gpu

CASES = {
    "one row": dict(length=[100], budget=[60]),
    "one position goes": dict(length=[100, 65], budget=[99, 64]),
    "all but one go": dict(length=[100, 17], budget=[1, 1]),
    "nothing stays": dict(length=[100, 1, 0], budget=[0, 0, 0]),
    "nothing goes": dict(length=[100, 1, 0], budget=[100, 5, 7]),
    "recent ones": dict(length=[300, 90, 64], budget=[200, 80, 60], recent=50),
    "all recent": dict(length=[300, 90, 20], budget=[200, 80, 10], recent=200),
    "recent ones that do not overlap": dict(length=[900], budget=[100], recent=90),
    "first ones": dict(length=[300, 90, 64], budget=[200, 80, 10], first=[150, 0, 30]),
    "first and recent exceed the budget": dict(length=[300, 90, 64], budget=[100, 20, 5], first=[90, 80, 64], recent=30),
    "negative first and budget": dict(length=[300, 90], budget=[-5, -1 << 31], first=[-7, -1 << 31], recent=3),
    "huge first, budget and recent": dict(length=[300, 90], budget=[(1 << 31) - 1, 4], first=[3, (1 << 31) - 1], recent=(1 << 31) - 1),
    "all equal": dict(length=[300, 1100], budget=[200, 1000], levels=1),
    "two weights": dict(length=[3000], budget=[1500], levels=2, recent=7, first=[5]),
    "long": dict(length=[9000, 40], budget=[4000, 30], levels=1 << 20, layers=1, page=64, recent=100),
    "many strips": dict(length=[5000, 1023, 1024, 1025, 1026], budget=[2500, 1000, 1000, 1000, 1025], levels=300, layers=1, kv_heads=1, first=[1, 0, 0, 1, 2], recent=1),
    "f32": dict(length=[300, 90, 64], budget=[200, 80, 60], recent=20, dtype="f32", head_dim=128, page=48),
    "narrow": dict(length=[300, 90, 64], budget=[200, 80, 60], recent=20, head_dim=8),
    "odd width": dict(length=[300, 90, 64], budget=[200, 80, 60], recent=21, head_dim=72, kv_heads=1),
    "f32, wide": dict(length=[300, 90], budget=[200, 80], recent=20, dtype="f32", head_dim=256),
    "memory by position": dict(length=[300, 90], budget=[200, 80], recent=20, order=(0, 1, 3, 2, 4)),
    "memory by page": dict(length=[300, 90], budget=[200, 80], recent=20, order=(1, 0, 2, 3, 4)),
    "large pages": dict(length=[3000, 900], budget=[1200, 1024], recent=20, page=1024),
    "very long": dict(length=[20000, 100], budget=[9000, 60], layers=1, kv_heads=2, page=64, recent=50, first=[7, 0], levels=1 << 20),
    "very long, many go": dict(length=[40000], budget=[300], layers=1, kv_heads=1, page=128, recent=299, levels=3),
    "very long, few go": dict(length=[17000], budget=[16990], layers=1, kv_heads=1, page=128, recent=300, levels=1 << 20),
    "very long, as bound": dict(length=[33, 70], budget=[20, 50], most=17000, recent=3),
    "sixteen thousand": dict(length=[16384, 4097], budget=[8000, 4000], layers=1, kv_heads=1, page=128, recent=10, levels=1 << 20),
    "sixteen thousand, equal": dict(length=[16384], budget=[8192], layers=1, kv_heads=1, page=128, levels=1),
    "four thousand, in order": dict(length=[4096, 4000], budget=[4000, 3990], layers=1, kv_heads=2, recent=2000, levels=1 << 20),
    "many rows": dict(length=[20 + 3 * i for i in range(70)], budget=[10 + i for i in range(70)], layers=1, kv_heads=1, recent=2),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name):
    kw = dict(CASES[name])
    print(f"[paged_evict] {name}: {kw}", flush=True)
    most = kw.pop("most", 0)
    p = Evict(list(CASES).index(name), kw.pop("length"), kw.pop("budget"), **kw, cap=most or None)
    p.args["max_seq_len"] = max(p.args["max_seq_len"], most)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("seed", range(16))
def test_random_shapes(seed):
    rng = np.random.default_rng(3000 + seed)
    rows = int(rng.integers(1, 9))
    most = int(rng.choice([30, 300, 2500]))
    kw = dict(length=[int(x) for x in rng.integers(0, most, rows)], budget=[int(x) for x in rng.integers(0, most, rows)], layers=int(rng.integers(1, 4)),
              kv_heads=int(rng.integers(1, 5)), head_dim=int(rng.choice([64, 128, 80])), page=int(rng.choice([16, 32, 48, 64, 256])), recent=int(rng.choice([0, 1, 20, most // 3])),
              first=None if rng.random() < 0.3 else [int(x) for x in rng.integers(0, most // 3, rows)], dtype=str(rng.choice(["bf16", "f32"])), levels=int(rng.choice([2, 30, 1 << 20])))
    print(f"[paged_evict] {kw}", flush=True)
    p = Evict(seed, kw.pop("length"), kw.pop("budget"), **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


def test_odd_weights():
    """Zeros of both signs are equal, NaN is less than everything, infinities are what they are."""
    p = Evict(20, [400, 64], [200, 30], recent=5, first=[3, 0], levels=3)
    rng = np.random.default_rng(1)
    mass = p.mass.cpu().numpy()
    for value in (-0.0, np.nan, np.inf, -np.inf, 1e-42, -1e-42, -3.0, 3.4e38):
        mass[rng.random(mass.shape) < 0.08] = value
    p.mass.copy_(torch.from_numpy(mass))
    p.was[2] = p.mass.clone()
    p.run()
    p.check()
    p = Evict(21, [400, 64], [200, 30])
    p.mass.fill_(float("nan"))
    p.was[2] = p.mass.clone()
    p.run()
    p.check()


def test_rows_that_break_their_bounds_stay_as_they_are():
    for change in (dict(seq_len=-1), dict(seq_len=301), dict(max_seq_len=299), dict(width=18), dict(cap=299)):
        print(f"[paged_evict] {change}", flush=True)
        p = Evict(22, [300, 90, 64], [200, 80, 60], recent=20)
        ctx = p.context()
        more = {}
        if "seq_len" in change:
            p.length = [change["seq_len"], 90, 64]
            more["seq_len"] = dev(p.length)
            p.args["max_seq_len"] = 300
        elif "max_seq_len" in change:
            more["max_seq_len"] = 299
        elif "width" in change:
            more["block_table"] = p.args["block_table"][:, :18]
        else:
            more.update(mass=p.mass[..., :299], mass_out=p.mass_out[..., :299])
        p.run(ctx, **more)
        assert ctx.device_status() == binding.ETREE
        p.check(skip=(0,))


def test_entries_outside_the_pool_set_the_flag():
    for entry in (-1, 1 << 30, -(1 << 31)):
        p = Evict(23, [300, 90], [200, 80], recent=20)
        table = p.args["block_table"].clone()
        table[0, 3] = entry
        ctx = p.context()
        p.run(ctx, block_table=table)
        assert ctx.device_status() == binding.ETREE
        assert p.args["seq_len_out"].tolist() == [200, 80]
        # the other row is whole
        others = p.table[1, :6]
        q = Evict(23, [300, 90], [200, 80], recent=20)
        q.run()
        assert torch.equal(p.k_pages[:, others], q.k_pages[:, others]) and torch.equal(p.mass_out, q.mass_out)


def test_lists_that_have_no_room():
    for free, capacity, count in ((3, 3, 3), (3, 30, -2), (3, 5, 6), (3, 5, 3)):
        p = Evict(24, [300, 90], [200, 40], recent=20)
        back = p.table[0, 13:19].tolist() + p.table[1, 3:6].tolist()
        ctx = p.context()
        lists = dev([-5] * capacity)
        p.run(ctx, free_pages=lists, free_count=dev([count]))
        base = min(max(count, 0), capacity)
        want = ([-5] * base + back + [-5] * capacity)[:capacity]
        assert lists.tolist() == want and p.args["free_count_out"].tolist() == [min(capacity, base + len(back))]
        fits = base == count and base + len(back) <= capacity
        assert (ctx.device_status() == binding.OK) == fits


def test_without_what_may_be_missing():
    p = Evict(25, [300, 90], [200, 80], recent=20)
    p.run(dropped=None, workspace=None)
    p.args["dropped"].copy_(dev([100, 10]))
    p.check()


def test_refusals():
    p = Evict(26, [300, 90], [200, 80], recent=20)
    ctx = p.context()
    keep = torch.empty(4096, dtype=torch.uint8, device="cuda")
    rec = binding._paged_evict_record(**p.args, workspace=keep)

    def call(**fields):
        a = binding.paged_evict_args.from_buffer_copy(rec)
        for k, v in fields.items():
            setattr(a, k, v)
        return ctx.lib.paged_evict(ctx.handle, C.byref(a))

    E = binding
    for k in ("seq_len", "budget", "mass", "mass_out", "k_pages", "v_pages", "block_table", "free_pages", "free_count", "free_count_out", "seq_len_out"):
        assert call(**{k: None}) == E.EINVAL, k
    for k in ("n_layers", "n_rows", "n_recent", "max_seq_len", "mass_cap", "free_capacity", "n_pages", "table_width", "workspace_bytes"):
        assert call(**{k: -1}) == E.EINVAL, k
    assert call(dtype=2) == E.EDTYPE
    for k, v in (("page_size", 24), ("head_dim", 4), ("stride_pos", 4), ("stride_layer", -8), ("n_rows", 3), ("max_seq_len", 301), ("mass_stride_head", 3), ("mass_stride_row", 3),
                 ("mass_stride_layer", 3)):
        assert call(**{k: v}) == E.ESHAPE, (k, v)
    for k, other in (("mass_out", "mass"), ("seq_len_out", "seq_len"), ("free_count_out", "free_count")):
        assert call(**{k: getattr(binding.paged_evict_args.from_buffer_copy(rec), other)}) == E.EINVAL, k
    for k in ("k_pages", "v_pages", "workspace"):
        assert call(**{k: getattr(binding.paged_evict_args.from_buffer_copy(rec), k) + 8}) == E.EINVAL, k
    assert call(n_rows=0) == E.OK and call(n_layers=0) == E.OK
    p = Evict(27, [17000], [200])
    ctx = p.context()
    rec = binding._paged_evict_record(**p.args, workspace=None)
    assert call(workspace=None) == E.EINVAL and call(workspace=keep.data_ptr(), workspace_bytes=64) == E.ESHAPE
    p = Evict(26, [300, 90], [200, 80], recent=20)
    torch.cuda.synchronize()
    assert torch.equal(p.k_pages.view(torch.int16), p.was[0].view(torch.int16)) and (p.mass_out == -7).all() and ctx.device_status() == E.OK
