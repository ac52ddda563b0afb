"""What the GPU tests of attention over pages reach: every kernel instance that the launch rules can choose is run by a test that compares its results (no GPU: the rules
are host code and are asked through the library)."""
import random

import test_gpu_paged_cuts as cuts
from paper_2605_07230_amd import binding


def test_every_cut_is_tested():
    reached, items = set(), set()      # (query rows, waves, head_dim, tree, keys in parts)
    for name, kw in cuts.CASES.items():
        for head_dim in (64, 128):
            rows, parts, waves = cuts.cut(name, head_dim)
            reached.add((rows, waves, head_dim, "tree" in kw, parts > 1))
            if rows == 16:             # more (row, kv head) pairs than workgroups that the chip holds: a workgroup takes several
                items.add((head_dim, "tree" in kw, len(kw["prefix"]) * kw["kv_heads"] * parts > 3 * 256))
    both = (False, True)
    few = {(16, 4, d, t, c) for d in (64, 128) for t in both for c in both} | {(16, 8, d, False, c) for d in (64, 128) for c in both}
    many = {(rows, 4, d, t, c) for rows in (64, 128) for d in (64, 128) for t in both for c in both} | {(256, 8, 64, t, c) for t in both for c in both}
    assert reached == few | many
    assert items == {(d, t, m) for d in (64, 128) for t in both for m in both}


def test_every_f32_cut_is_tested():
    reached = {(head_dim, *cuts.f32_cut(name, head_dim)[1:]) for name in cuts.F32 for head_dim in (64, 100, 251)}
    assert {(d, w) for d, p, w in reached if p == 1} == {(d, w) for d, p, w in reached if p > 1} == {(64, 16), (100, 8), (251, 4)}


def test_no_call_takes_256_rows_at_head_dim_128():
    """The launch has no such kernel."""
    rng = random.Random(3)
    for _ in range(3000):
        rows, new = int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 12))
        kv, group, tree = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 3, 8]), rng.random() < 0.5
        cut = binding.paged_cut(n_rows=rows, n_tokens=rng.randint(new, rows * new), max_new=new, max_prefix_len=int(2 ** rng.uniform(0, 16)) - 1, n_heads=kv * group,
                                n_kv_heads=kv, head_dim=128, tree=tree, window=rng.choice([0, 0, 300]))
        assert cut[0] in (16, 64, 128)


def test_the_query_refuses_what_it_does_not_describe():
    lib, n, a = binding.load_library(), binding.C.c_int32(), binding.paged_attn_args()
    assert lib.cascade_paged_cut(None, None, n, n, n) == binding.EINVAL and lib.cascade_paged_cut(None, a, n, n, None) == binding.EINVAL
    assert lib.cascade_paged_cut(None, a, n, n, n) == binding.EINVAL           # no rows
    a.dtype = 7
    assert lib.cascade_paged_cut(None, a, n, n, n) == binding.EDTYPE
    good = dict(n_rows=1, n_tokens=1, max_new=1, n_heads=2, n_kv_heads=1, head_dim=64, dtype=binding.BF16)
    for changes in ({}, dict(dtype=binding.F32, head_dim=3)):
        b = binding.paged_attn_args(**{**good, **changes})
        assert lib.cascade_paged_cut(None, b, n, n, n) == binding.OK
    for k, v in (("n_rows", 0), ("n_tokens", -1), ("max_new", 2 ** 31 - 1), ("max_prefix_len", 2 ** 31 - 1), ("max_prefix_len", -1), ("window", -1), ("n_sink", -1), ("n_kv_heads", 0),
                 ("n_heads", 0), ("head_dim", 96)):
        assert lib.cascade_paged_cut(None, binding.paged_attn_args(**{**good, k: v}), n, n, n) == binding.EINVAL, k
