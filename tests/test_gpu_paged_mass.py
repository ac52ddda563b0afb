"""paged_mass against the oracle: lengths, page sizes, orders of memory, windows, accepted paths, both types; what counts nothing; refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding

from budget_util import Mass
from serving_util import dev

pytestmark = pytest.mark.gpu

CASES = {
    "one token, alone": dict(length=[1], new=[1]),
    "one token": dict(length=[313, 313], new=[1, 1], heads=32, kv_heads=32),
    "lengths around tiles and pages": dict(length=[1, 2, 16, 17, 18, 64, 65, 66, 255, 256, 257, 258], new=[1] * 12, heads=4, kv_heads=2),
    "few tokens, grouped": dict(length=[703, 20, 2, 65], new=[3, 17, 2, 1], heads=16, kv_heads=2),
    "one kv head of 8": dict(length=[1001, 91], new=[1, 1], heads=8, kv_heads=1, page=32),
    "group of 3": dict(length=[501, 86, 33], new=[1, 9, 33], heads=12, kv_heads=4, page=48),
    "group of 20": dict(length=[501, 79, 5], new=[1, 2, 5], heads=20, kv_heads=1),
    "rows without tokens": dict(length=[50, 65, 0, 71], new=[0, 5, 0, 1]),
    "prompts": dict(length=[300, 257, 16], new=[300, 257, 16], heads=8, kv_heads=2),
    "chunks behind some": dict(length=[900, 700, 1100], new=[100, 333, 64], heads=4, kv_heads=4, page=128),
    "a long chunk": dict(length=[2100], new=[1000], heads=4, kv_heads=1, page=64),
    "long, one token": dict(length=[9001], new=[1], heads=4, kv_heads=1, page=1024),
    "narrow heads": dict(length=[230, 701, 129], new=[130, 1, 64], heads=8, kv_heads=2, head_dim=64),
    "memory by position": dict(length=[170, 260], new=[70, 1], order="position"),
    "memory by head": dict(length=[170, 260], new=[70, 1], order="page_inside"),
    "slices of one projection": dict(length=[170, 260], new=[70, 1], packed=True, spare=5),
    "paths": dict(length=[613, 1005, 40, 7], new=[11, 1, 5, 7], path=60),
    "paths, positions left out": dict(length=[613, 1005, 400, 330], new=[11, 1, 5, 7], path=60, first=[304, 304, 304, 304]),
    "everything left out": dict(length=[613, 100], new=[11, 1], first=[613, 5000]),
    "first inside a group": dict(length=[613, 100], new=[300, 1], first=[37, -4]),
    "window": dict(length=[401, 91, 1001], new=[1, 1, 1], window=100, n_sink=4),
    "window of one": dict(length=[405, 3], new=[5, 3], window=1),
    "window, chunk": dict(length=[1000, 333, 41], new=[300, 333, 1], heads=4, kv_heads=2, window=64, n_sink=3),
    "window, many sinks": dict(length=[1000], new=[100], heads=2, kv_heads=1, window=130, n_sink=200, head_dim=64),
    "window wider than all": dict(length=[150, 8], new=[50, 1], window=5000, n_sink=1),
    "window and first": dict(length=[1000, 700], new=[40, 3], window=300, n_sink=20, first=[7, 690]),
    "scale": dict(length=[315, 50], new=[3, 40], scale=0.03),
}
F32 = {
    "f32": dict(length=[271, 15], new=[15, 15], heads=8, kv_heads=8, head_dim=64),
    "f32 odd head": dict(length=[103, 20, 18], new=[3, 20, 1], heads=4, kv_heads=2, head_dim=70),
    "f32 wide head": dict(length=[130, 34], new=[30, 1], heads=4, kv_heads=4, head_dim=256),
    "f32 head of 3": dict(length=[45], new=[5], heads=2, kv_heads=1, head_dim=3),
    "f32 head of 100": dict(length=[445, 90], new=[5, 60], heads=4, kv_heads=2, head_dim=100),
    "f32 odd wide head": dict(length=[200], new=[70], heads=4, kv_heads=2, head_dim=201, packed=True),
    "f32 window": dict(length=[400, 21, 90], new=[100, 1, 90], heads=4, kv_heads=2, head_dim=80, window=30, n_sink=3),
    "f32 path": dict(length=[700, 300], new=[11, 4], heads=4, kv_heads=2, head_dim=64, path=40, first=[100, 0]),
}


@pytest.mark.parametrize("name", [*CASES, *F32])
def test_against_the_oracle(name):
    kw = dict(CASES.get(name) or dict(F32[name], dtype="f32"))
    print(f"[paged_mass] {name}: {kw}", flush=True)
    p = Mass(list([*CASES, *F32]).index(name), kw.pop("length"), kw.pop("new"), **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("seed", range(20))
def test_random_shapes(seed):
    rng = np.random.default_rng(2000 + seed)
    rows = int(rng.integers(1, 9))
    kv = int(rng.choice([1, 2, 4]))
    new = [int(x) for x in rng.integers(0, rng.choice([2, 20, 300]), rows)]
    new[0] = max(new[0], 1)
    kw = dict(length=[n + int(x) for n, x in zip(new, rng.integers(0, rng.choice([20, 300, 1500]), rows))], new=new, heads=kv * int(rng.choice([1, 2, 4, 5])), kv_heads=kv,
              head_dim=int(rng.choice([64, 128])), page=int(rng.choice([16, 32, 48, 64, 256])), order=str(rng.choice(["head", "position", "page_inside"])),
              dtype="f32" if seed % 6 == 5 else "bf16", path=int(rng.choice([0, 0, 33])), spare=int(rng.integers(0, 3)))
    if rng.random() < 0.4:
        kw.update(window=int(rng.integers(1, 400)), n_sink=int(rng.integers(0, 90)))
    if rng.random() < 0.4:
        kw.update(first=[int(x) for x in rng.integers(0, 200, rows)])
    print(f"[paged_mass] {kw}", flush=True)
    p = Mass(seed, kw.pop("length"), kw.pop("new"), **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("rows", [2, 3, 16, 17, 64, 65, 70])
@pytest.mark.parametrize("most", [1, 40, 300])
def test_rows_of_all_lengths(rows, most):
    """Blocks of keys are dealt to workgroups by the rows' lengths: equal ones, rows without tokens, the longest one last, rows of one position."""
    rng = np.random.default_rng(rows * 1000 + most)
    new = [int(x) for x in rng.integers(0, most + 1, rows)]
    new[0] = new[rows // 2] = most
    length = [n + int(x) for n, x in zip(new, rng.integers(0, 700, rows))]
    length[-1], new[-1] = 1300, most
    if rows > 2:
        length[1] = new[1] = 1
        length[rows // 2] = length[0]
    p = Mass(rows + most, length, new, heads=4, kv_heads=2, head_dim=64 if rows % 2 else 128, path=0)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_that_count_nothing(dtype):
    """Without a finite lse, or without a source."""
    for kw in (dict(length=[300, 40], new=[70, 3]), dict(length=[300, 40], new=[70, 3], path=20)):
        p = Mass(5, heads=4, kv_heads=2, dtype=dtype, **kw)
        at = torch.from_numpy(p.source[[0, 13, 30, 71]]).cuda()
        for i, value in enumerate((float("inf"), -float("inf"), float("nan"), float("inf"))):
            p.lse[at[i], 1 + i % 2] = value
        if p.args["source"] is not None:
            p.args["source"][[5, 72]] = -1
            # as tokens whose lse is none
            lse = p.lse.clone()
            p.lse[torch.from_numpy(p.source[[5, 72]]).cuda()] = -float("inf")
            ctx = p.context()
            p.run(ctx, lse=lse)
        else:
            ctx = p.context()
            p.run(ctx)
        assert ctx.device_status() == binding.OK
        p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_keys_that_a_token_does_not_attend_do_not_reach_the_sums(dtype, value):
    """Such a key shows at its own position and nowhere else."""
    for kw in (dict(length=[300, 40], new=[70, 3]), dict(length=[300, 40], new=[70, 3], window=20, n_sink=2)):
        p = Mass(6, heads=4, kv_heads=2, dtype=dtype, **kw)
        for y in (299, 250):
            p.k_pages[p.table[0, y // 16], 1, y % 16, 5] = float("nan")
        p.run()
        p.check()
        # with lse that is infinite for the tokens that meet an infinite score, as attention leaves it
        p = Mass(6, heads=4, kv_heads=2, dtype=dtype, **kw)
        p.k_pages[p.table[0, 299 // 16], 1, 299 % 16, 5] = value
        p.lse[69, 2:] = value
        p.run()
        p.check()


def test_rows_that_break_their_bounds_stay_as_they_are():
    for change in (dict(seq_len=[2, 52]), dict(seq_len=[-3, 52]), dict(seq_len=[1 << 30, 52]), dict(max_new=2), dict(q_off=[0, 9, 5]), dict(q_off=[-1, 3, 5]), dict(max_seq_len=42),
                   dict(width=2), dict(cap=42)):
        for dtype in ("bf16", "f32"):
            print(f"[paged_mass] {change} {dtype}", flush=True)
            p = Mass(8, [43, 42 if "max_seq_len" in change or "cap" in change else 32], [3, 2], heads=4, kv_heads=2, dtype=dtype)
            more = dict(change)
            if "width" in change:
                more = dict(block_table=p.args["block_table"][:, :2])
            elif "cap" in change:
                more = dict(mass=p.mass[:, :, :42])
            for k in ("seq_len", "q_off"):
                if k in more:
                    more[k] = dev(more[k])
            ctx = p.context()
            if isinstance(change.get("seq_len"), list):
                more["seq_len"][1] = p.length[1]
            p.run(ctx, **more)
            assert ctx.device_status() == binding.ETREE
            bad = [0, 1] if change.get("q_off") == [0, 9, 5] else [0]
            for s in bad:
                assert torch.equal(p.mass[s].nan_to_num(-1), p.before[s].nan_to_num(-1)), change
            if "q_off" not in change:
                p.check(rows=[1])
            assert ctx.device_status() == binding.OK


@pytest.mark.parametrize("rows", [4, 20, 70])
@pytest.mark.parametrize("tokens", [1, 90])
def test_one_of_many_that_breaks_its_bounds(rows, tokens):
    for bad, value in ((0, -1), (2, 1 << 30), (rows - 1, tokens - 1)):
        p = Mass(rows + bad, [tokens + 37 * (s % 7) for s in range(rows)], [tokens] * rows, heads=4, kv_heads=2)
        lengths = list(p.length)
        lengths[bad] = value
        ctx = p.context()
        p.run(ctx, seq_len=dev(lengths))
        assert ctx.device_status() == binding.ETREE
        assert torch.equal(p.mass[bad].nan_to_num(-1), p.before[bad].nan_to_num(-1))
        p.check(rows=[s for s in range(rows) if s != bad])
        assert ctx.device_status() == binding.OK


def test_entries_and_sources_outside_set_the_flag():
    for entry in (-1, 1 << 30, -(1 << 31)):
        for dtype in ("bf16", "f32"):
            p = Mass(9, [300, 52], [100, 2], heads=4, kv_heads=2, dtype=dtype)
            table = p.args["block_table"].clone()
            table[0, 4] = entry
            p.table[0, 4] = entry
            ctx = p.context()
            p.run(ctx, block_table=table)
            assert ctx.device_status() == binding.ETREE
            p.check()
    p = Mass(9, [300, 52], [100, 2], heads=4, kv_heads=2, path=10)
    p.args["source"][7] = 112
    p.args["source"][8] = -2
    p.lse[torch.from_numpy(p.source[[7, 8]]).cuda()] = float("nan")
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.ETREE
    p.check()


def test_rows_that_got_no_room_stay_as_they_are():
    for dtype, new in (("bf16", [3, 2]), ("bf16", [40, 30]), ("f32", [3, 2])):
        p = Mass(12, [243, 252], new, heads=4, kv_heads=2, dtype=dtype)
        ctx = p.context()
        p.run(ctx, prefix_len=dev([243, 252 - new[1]]))
        assert ctx.device_status() == binding.OK
        assert torch.equal(p.mass[0].nan_to_num(-1), p.before[0].nan_to_num(-1))
        p.check(rows=[1])
        p.run(ctx, prefix_len=dev([243 - new[0], 251]))
        assert ctx.device_status() == binding.ETREE
        p.check(rows=[0])


def test_sums_repeat():
    p = Mass(10, [1500, 700], [300, 1], heads=8, kv_heads=2)
    ctx = p.context()
    p.run(ctx)
    first = p.mass.clone()
    p.mass.copy_(p.before)
    p.run(ctx)
    assert torch.equal(first, p.mass)


def test_refusals():
    p = Mass(11, [43, 52], [3, 2], heads=4, kv_heads=2)
    ctx = p.context()
    seen = []
    real = ctx.lib.paged_mass_record
    ctx.lib.paged_mass_record = lambda handle, rec: seen.append(rec) or 0
    try:
        binding.paged_mass(ctx, **p.args)
    finally:
        ctx.lib.paged_mass_record = real

    def call(**fields):
        a = binding.paged_mass_args.from_buffer_copy(seen[0])
        for k, v in fields.items():
            setattr(a, k, v)
        return ctx.lib.paged_mass(ctx.handle, C.byref(a))

    E = binding
    for k in ("q_off", "seq_len", "q", "lse", "k_pages", "block_table", "mass"):
        assert call(**{k: None}) == E.EINVAL, k
    for k in ("n_rows", "n_tokens", "n_source", "max_new", "max_seq_len", "window", "n_sink", "mass_cap", "n_pages", "table_width"):
        assert call(**{k: -1}) == E.EINVAL, k
    assert call(dtype=2) == E.EDTYPE and call(scale=float("nan")) == E.EINVAL and call(n_source=4) == E.EINVAL
    for k, v in (("page_size", 24), ("n_heads", 5), ("n_heads", 8), ("head_dim", 96), ("stride_pos", 4), ("stride_head", -8), ("q_stride", 8), ("n_rows", 3), ("n_tokens", 6),
                 ("max_seq_len", 53), ("max_new", 0), ("max_seq_len", 0), ("mass_stride_head", 3), ("mass_stride_row", 3)):
        got = call(**{k: v})
        assert got == (E.EINVAL if (k, v) == ("n_tokens", 6) else E.ESHAPE), (k, v, got)
    for k in ("q", "k_pages"):
        assert call(**{k: getattr(binding.paged_mass_args.from_buffer_copy(seen[0]), k) + 8}) == E.EINVAL, k
    assert call(n_rows=0) == E.OK and call(n_tokens=0) == E.OK
    torch.cuda.synchronize()
    assert torch.equal(p.mass.nan_to_num(-1), p.before.nan_to_num(-1)) and ctx.device_status() == E.OK
