"""paged_slots and paged_append against the oracle, and a commit to pages against kv_commit's."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding

from serving_util import DT, ORDERS, dev

pytestmark = pytest.mark.gpu


def _context(rows, tokens=4096, stream=None):
    return binding.Context(max_rows=rows, max_nodes_total=tokens, max_nodes_per_tree=1, max_prefix=1, n_heads=1, head_dim=64, hidden=64, vocab=64, stream=stream)


def _slots(ctx, seq, new, table, free, page, n_pages, tokens, free_count=None, width=None, **path):
    rows = len(seq)
    one = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
    block = dev(table)
    got = dict(q_off=one(rows + 1), slot_map=one(tokens), position=one(tokens), source=one(tokens), seq_len_out=one(rows), free_count_out=one(1))
    binding.paged_slots(ctx, seq_len=dev(seq), new_len=None if new is None else dev(new), block_table=block[:, :width], free_pages=dev(free),
                        free_count=dev([len(free) if free_count is None else free_count]), page_size=page, n_pages=n_pages, **got, **path)
    torch.cuda.synchronize()
    return {**{k: v.cpu().numpy() for k, v in got.items()}, "table": block.cpu().numpy()}


def _same(got, want):
    for k in ("q_off", "slot_map", "position", "source", "table"):
        assert np.array_equal(got[k], want[k]), (k, np.argwhere(got[k] != want[k])[:5])
    assert np.array_equal(got["seq_len_out"], want["seq_len"]) and int(got["free_count_out"][0]) == want["free_count"]


def _tables(rng, seq, page, width, extra):
    held = [-(-int(x) // page) if x > 0 else 0 for x in seq]
    ids = rng.permutation(sum(held) + extra)
    table, at = np.full((len(seq), width), -5, np.int64), 0
    for s, h in enumerate(held):
        table[s, :h] = ids[at:at + h]
        at += h
    return table, ids[at:], len(ids)


@pytest.mark.parametrize("rows,most_seq,most_new,page", [(1, 1, 1, 16), (1, 500, 300, 16), (5, 40, 3, 32), (64, 600, 1, 16), (300, 100, 90, 48), (257, 30, 5, 1024),
                                                         (3, 0, 5000, 64), (700, 20, 1, 16)])
def test_slots(rows, most_seq, most_new, page):
    print(f"[paged_slots] {rows} rows, {most_seq}, {most_new}, pages of {page}", flush=True)
    rng = np.random.default_rng(rows + page)
    seq, new = rng.integers(0, most_seq + 1, rows), rng.integers(0, most_new + 1, rows)
    width = -(-(most_seq + most_new) // page) + 1
    table, free, pool = _tables(rng, seq, page, width, rows * width)
    ctx = _context(rows)
    tokens = int(new.sum()) + int(rng.integers(0, 600))
    got = _slots(ctx, seq, new, table, free, page, pool, tokens)
    _same(got, so.paged_slots(seq, new, table, free, len(free), page, tokens))
    assert ctx.device_status() == binding.OK


@pytest.mark.parametrize("seed", range(6))
def test_slots_without_room(seed):
    """Too few pages, tables or places, lengths below zero: those rows keep what they have, the flag is set."""
    rng = np.random.default_rng(seed)
    rows, page, width = int(rng.integers(1, 400)), 16, 6
    seq, new = rng.integers(0, 60, rows), rng.integers(0, 60, rows)
    table, free, pool = _tables(rng, seq, page, width, 40)
    if seed % 2:
        new[rng.integers(0, rows)] = -3
        new[rng.integers(0, rows)] = 2 ** 31 - 1
    if seed % 3 == 0:
        seq[rng.integers(0, rows)] = -1
    tokens = int(min(np.maximum(new, 0).sum(), 3000) * (0.7 if seed > 2 else 1)) + 1
    print(f"[paged_slots] short {seed}: {rows} rows, {tokens} places", flush=True)
    ctx = _context(rows)
    want = so.paged_slots(seq, new, table, free, len(free), page, tokens)
    got = _slots(ctx, seq, new, table, free, page, pool, tokens)
    _same(got, want)
    assert ctx.device_status() == (binding.ETREE if want["refused"].any() else binding.OK)


def test_slots_with_bad_pages_and_counts():
    ctx = _context(2)
    # a count above the list's length is the list's length; below zero none
    got = _slots(ctx, [0, 0], [3, 3], np.full((2, 2), -5), [0, 1], 16, 2, 6, free_count=9)
    assert got["free_count_out"][0] == 0 and got["slot_map"].tolist() == [16, 17, 18, 0, 1, 2] and ctx.device_status() == binding.ETREE
    got = _slots(ctx, [0, 0], [3, 3], np.full((2, 2), -5), [0, 1], 16, 2, 6, free_count=-9)
    assert got["free_count_out"][0] == 0 and (got["slot_map"] == -1).all() and ctx.device_status() == binding.ETREE
    # a page outside the pool, in the list and in the table
    got = _slots(ctx, [0, 0], [3, 3], np.full((2, 2), -5), [7, 1], 16, 2, 6)
    assert got["slot_map"].tolist() == [16, 17, 18, -1, -1, -1] and got["table"].tolist() == [[1, -5], [-1, -5]] and ctx.device_status() == binding.ETREE
    got = _slots(ctx, [2, 0], [3, 3], np.array([[9, -5], [-5, -5]]), [0, 1], 16, 2, 6)
    assert got["slot_map"].tolist() == [-1, -1, -1, 16, 17, 18] and ctx.device_status() == binding.ETREE


def _paths(rng, prompts, depth, nodes):
    accept = rng.integers(0, depth + 1, prompts)
    path = np.full((prompts, depth), -1)
    for b in range(prompts):
        path[b, :accept[b]] = np.sort(rng.choice(np.arange(1, nodes), accept[b], replace=False))
    return accept, path


@pytest.mark.parametrize("prompts,depth,page", [(1, 3, 16), (8, 10, 16), (40, 64, 32), (150, 5, 16)])
def test_slots_of_accepted_paths(prompts, depth, page):
    print(f"[paged_slots] paths of {prompts} prompts, {depth}", flush=True)
    rng = np.random.default_rng(prompts)
    rows, nodes = 2 * prompts, depth + 20
    accept, path = _paths(rng, prompts, depth, nodes)
    row_prompt = np.repeat(np.arange(prompts), 2)
    seq = rng.integers(0, 300, rows)
    table, free, pool = _tables(rng, seq, page, 30, rows * 6)
    off = np.arange(rows + 1) * nodes
    new = 1 + accept[row_prompt]
    source = [[off[s]] + [off[s] + x for x in path[row_prompt[s], :new[s] - 1]] for s in range(rows)]
    tokens = rows * (depth + 1)
    ctx = _context(rows, rows * nodes)
    more = dict(node_off=dev(off), row_prompt=dev(row_prompt), accept_len=dev(accept), path_nodes=dev(path), n_nodes_total=rows * nodes)
    _same(_slots(ctx, seq, None, table, free, page, pool, tokens, **more), so.paged_slots(seq, new, table, free, len(free), page, tokens, source))
    assert ctx.device_status() == binding.OK
    # a path entry outside the tree, a prompt and an accepted length that do not exist
    path[0, 0], accept[0] = nodes, 1
    new = 1 + accept[row_prompt]
    row_prompt[-1] = prompts
    new[-1] = 0
    if prompts > 1:
        accept[1] = depth + 1
        new[2:4] = 0
    source = [[off[s]] + [off[s] + x if x < nodes else -1 for x in path[min(row_prompt[s], prompts - 1), :max(new[s] - 1, 0)]] for s in range(rows)]
    more.update(path_nodes=dev(path), accept_len=dev(accept), row_prompt=dev(row_prompt))
    got, want = _slots(ctx, seq, None, table, free, page, pool, tokens, **more), so.paged_slots(seq, new, table, free, len(free), page, tokens, source)
    _same(got, want)
    assert ctx.device_status() == binding.ETREE


@pytest.mark.parametrize("dtype,layers,tokens,heads,head_dim,page,order", [
    ("bf16", 1, 1, 1, 64, 16, "head"), ("bf16", 30, 16, 8, 128, 16, "head"), ("f32", 3, 77, 2, 20, 32, "position"), ("bf16", 2, 500, 4, 72, 48, "page_inside"),
    ("bf16", 5, 63, 3, 8, 1024, "position"), ("f32", 1, 2000, 1, 4, 16, "head")])
def test_append(dtype, layers, tokens, heads, head_dim, page, order):
    print(f"[paged_append] {dtype} {layers} {tokens} {heads} {head_dim} {page} {order}", flush=True)
    rng = np.random.default_rng(tokens)
    n_pages = -(-tokens // page) + 5
    slot = rng.permutation(n_pages * page)[:tokens]
    slot[rng.random(tokens) < 0.2] = -1
    perm = ORDERS[order]
    shape = (n_pages, heads, page, head_dim)
    pools = [torch.randn(layers, *(shape[i] for i in perm), device="cuda").to(DT[dtype]).permute(0, *(1 + np.argsort(perm))) for _ in range(2)]
    for with_source in (False, True):
        n_source = tokens + 9 if with_source else tokens
        new = [torch.randn(layers, n_source, heads, head_dim, device="cuda").to(DT[dtype]) for _ in range(2)]
        source = rng.integers(0, n_source, tokens) if with_source else np.arange(tokens)
        want = [p.clone() for p in pools]
        ok = slot >= 0
        for w, x in zip(want, new):
            w[:, dev(slot[ok] // page, np.int64), :, dev(slot[ok] % page, np.int64)] = x[:, dev(source[ok], np.int64)].transpose(0, 1)
        ctx = _context(1)
        binding.paged_append(ctx, k_new=new[0], v_new=new[1], slot_map=dev(slot), source=dev(source) if with_source else None, k_pages=pools[0], v_pages=pools[1])
        torch.cuda.synchronize()
        assert ctx.device_status() == binding.OK
        for p, w in zip(pools, want):
            assert torch.equal(p, w)
    # slots and sources that do not exist are skipped and flagged
    before = [p.clone() for p in pools]
    for bad_slot, bad_source in ((n_pages * page, 0), (-2, 0), (3, tokens), (3, -1)):
        binding.paged_append(ctx, k_new=new[0], v_new=new[1], slot_map=dev([bad_slot]), source=dev([bad_source if bad_source != tokens else n_source]), k_pages=pools[0],
                             v_pages=pools[1])
        assert ctx.device_status() == binding.ETREE
    assert all(torch.equal(a, b) for a, b in zip(before, pools))


def test_append_past_32_bits():
    """A pool whose places lie further apart than 32 bits count bytes."""
    pool = torch.empty(1, 40000, 8, 64, 128, dtype=torch.bfloat16, device="cuda")          # 5.2 GB
    new = torch.randn(1, 3, 8, 128, device="cuda").to(torch.bfloat16)
    slots = [39999 * 64 + 63, 20000 * 64, 7]
    print("[paged_append] 5 GB pool", flush=True)
    ctx = _context(1)
    binding.paged_append(ctx, k_new=new, v_new=new, slot_map=dev(slots), k_pages=pool, v_pages=pool)
    torch.cuda.synchronize()
    for t, slot in enumerate(slots):
        assert torch.equal(pool[0, slot // 64, :, slot % 64], new[0, t])
    q, out = torch.randn(1, 8, 128, device="cuda").to(torch.bfloat16), torch.empty(1, 8, 128, device="cuda", dtype=torch.bfloat16)
    # attention reads there as well: one cached position, in the last page
    pool[0, 39999, :, 0] = new[0, 1]
    big = binding.Context(max_rows=1, max_nodes_total=1, max_nodes_per_tree=1, max_prefix=1, n_heads=8, head_dim=128, hidden=64, vocab=64)
    binding.paged_attn(big, q_off=dev([0, 1]), prefix_len=dev([1]), block_table=dev([[39999]]), q=q, k_new=new[0, :1], v_new=new[0, :1], k_pages=pool[0], v_pages=pool[0],
                       out=out, max_new=1, max_prefix_len=1)
    k = torch.stack([new[0, 1], new[0, 0]]).double()                                        # [2, 8, 128]
    w = torch.softmax((q[0].double()[None] * k).sum(-1) / 128 ** 0.5, 0)
    ref = (w[..., None] * k).sum(0)
    assert ((out[0].double() - ref).abs() <= 3 * 2.0 ** -8 * (w[..., None] * k.abs()).sum(0) + 1e-6).all()


def test_refusals_of_slots_and_append():
    ctx = _context(2, 8)
    E = binding
    t = [torch.zeros(8, dtype=torch.int32, device="cuda") for _ in range(9)]
    rec = binding._SLOTS(2, 16, 4, 2, 2, 8, 4, t[0].data_ptr(), t[1].data_ptr(), 0, 0, 0, 0, 0, 0, 0, *[x.data_ptr() for x in t[2:]], 0, 0)
    base = dict(position=None, source=None, seq_len_out=torch.zeros(2, dtype=torch.int32, device="cuda").data_ptr())

    def slots(**fields):
        a = binding.paged_slots_args.from_buffer_copy(rec)
        for k, v in {**base, **fields}.items():
            setattr(a, k, v)
        return ctx.lib.paged_slots(ctx.handle, C.byref(a))

    a = binding.paged_slots_args.from_buffer_copy(rec)
    for k in ("seq_len", "block_table", "free_pages", "free_count", "free_count_out", "q_off", "slot_map", "seq_len_out"):
        assert slots(**{k: None}) == E.EINVAL, k
    assert slots(seq_len_out=a.seq_len) == E.EINVAL and slots(free_count_out=a.free_count) == E.EINVAL
    for k in ("n_rows", "table_width", "max_tokens", "free_capacity", "n_pages", "page_size"):
        assert slots(**{k: -1}) == E.EINVAL, k
    assert slots(table_stride=1) == E.EINVAL and slots(page_size=0) == E.EINVAL
    for k, v in (("page_size", 8), ("page_size", 1040), ("n_rows", 3), ("n_pages", 1 << 27), ("table_width", 1 << 27)):
        assert slots(**{k: v}, **({"table_stride": 1 << 28} if k == "table_width" else {})) == E.ESHAPE, (k, v)
    assert slots(new_len=None) == E.EINVAL                      # neither lengths nor paths
    path = dict(new_len=None, node_off=a.q_off, row_prompt=a.q_off, accept_len=a.q_off, path_nodes=a.q_off, source=a.slot_map, n_prompts=1, max_depth=3, n_nodes_total=4)
    for k in ("node_off", "row_prompt", "accept_len", "path_nodes", "source"):
        assert slots(**{**path, k: None}) == E.EINVAL, k
    assert slots(**{**path, "max_depth": 65}) == E.ESHAPE and slots(**{**path, "n_nodes_total": 9}) == E.ESHAPE
    assert slots(n_rows=0) == E.OK

    pool = torch.full((1, 2, 2, 16, 64), 3.0, device="cuda")
    rec2 = binding._APPEND(0, 1, 2, 2, 2, 64, t[0].data_ptr(), 0, pool.data_ptr(), pool.data_ptr(), pool.data_ptr(), pool.data_ptr(), 4096, 2048, 1024, 64, 2, 16)

    def append(**fields):
        a = binding.paged_append_args.from_buffer_copy(rec2)
        for k, v in fields.items():
            setattr(a, k, v)
        return ctx.lib.paged_append(ctx.handle, C.byref(a))

    for k in ("slot_map", "k_new", "v_new", "k_pages", "v_pages"):
        assert append(**{k: None}) == E.EINVAL, k
    for k in ("n_layers", "n_tokens", "n_source", "n_kv_heads", "head_dim", "n_pages", "page_size"):
        assert append(**{k: -1}) == E.EINVAL, k
    assert append(dtype=7) == E.EDTYPE and append(n_source=1) == E.EINVAL and append(k_pages=pool.data_ptr() + 4) == E.EINVAL
    for k, v in (("head_dim", 6), ("stride_page", 2), ("stride_pos", -4), ("page_size", 20), ("n_layers", 70000), ("n_tokens", 2 ** 31 - 1)):
        assert append(**{k: v}, **({"n_source": 2 ** 31 - 1} if k == "n_tokens" else {})) == E.ESHAPE, (k, v)
    assert append(n_tokens=0) == E.OK and append(n_layers=0) == E.OK
    torch.cuda.synchronize()
    assert (pool == 3).all() and ctx.device_status() == E.OK
