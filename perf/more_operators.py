"""Operators for a cache in pages that rows share and that is held to a budget: what they are timed on, how inputs are made, and one pass through each.

``shared``  attention of new tokens of rows whose first positions lie in the same pages: those are read once for a group of rows
``mass``    the attention weight that cached positions gather, per row and kv head
``evict``   rows that have outgrown their budget keep their heaviest positions; the pages behind go back

Where ``own`` is false a pass is written in elementary torch operations, in 32 bits; where it is true it is the call of
``paper_2605_07230_amd.binding`` that a serving program makes.  Sizes are the repository's own configurations (``workloads.make_config``, ``bench.py``) and the
ranges between them, and longer prefixes where many rows share them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

SHARED = dict(kind="shared", dtype="bf16", rows=8, groups=1, heads=32, kv_heads=32, head_dim=128, shared_min=304, shared_max=304, own_min=0, own_max=300,
              new_min=1, new_max=1, page=16, tree=False, depth=0, shape_seed=0)
MASS = dict(kind="mass", dtype="bf16", rows=2, heads=32, kv_heads=32, head_dim=128, prefix_min=312, prefix_max=312, new_min=1, new_max=1, page=16, window=0,
            sinks=0, path=False, first=0, shape_seed=0)
EVICT = dict(kind="evict", dtype="bf16", layers=1, rows=2, kv_heads=32, head_dim=128, len_min=400, len_max=600, budget_min=312, budget_max=312, first_max=4,
             recent=32, page=16, shape_seed=0)


def listed():
    return [
        # eight images of one prompt, a token each, early in their images: latency
        dict(SHARED, name="shared_token"),
        # a full batch behind one long prefix, grouped heads: the rows' own keys stream, the shared ones are products
        dict(SHARED, name="shared_token_batch", rows=64, kv_heads=8, shared_min=4192, shared_max=4192, own_min=90, own_max=600, page=32, shape_seed=1),
        # prefixes much longer than the images, groups of different sizes (rows of their own among them), a few tokens to a row, narrow heads
        dict(SHARED, name="shared_long", rows=48, groups=6, heads=16, kv_heads=4, head_dim=64, shared_min=500, shared_max=16384, own_min=1, own_max=2000,
             new_min=1, new_max=4, page=64, shape_seed=2),
        # verification of 60-node trees of sixteen rows, two prompts
        dict(SHARED, name="shared_trees", rows=16, groups=2, shared_min=1200, shared_max=2048, own_min=100, own_max=500, new_min=60, new_max=60, tree=True,
             depth=6, page=16, shape_seed=3),
        # the fp32 configuration: fifteen new tokens of six rows
        dict(SHARED, name="shared_f32", dtype="f32", rows=6, heads=8, kv_heads=8, head_dim=64, shared_min=256, shared_max=256, own_min=1, own_max=100, new_min=15,
             new_max=15, tree=True, depth=5, shape_seed=4),
        # a token of one user and the guidance row: latency
        dict(MASS, name="mass_token"),
        # a full batch, anywhere in the images: the keys stream
        dict(MASS, name="mass_token_batch", rows=64, kv_heads=8, prefix_min=90, prefix_max=4200, page=32, shape_seed=1),
        # chunks of prompts, ragged: products and exponentials bound it
        dict(MASS, name="mass_chunks", rows=8, kv_heads=8, prefix_min=0, prefix_max=2000, new_min=500, new_max=1000, page=64, shape_seed=2),
        # what a verification step kept: paths of up to ten nodes out of trees, positions of a shared prompt left out
        dict(MASS, name="mass_path", rows=16, prefix_min=600, prefix_max=2356, new_min=1, new_max=11, path=True, first=304, shape_seed=3),
        # one layer of one user and the guidance row: latency
        dict(EVICT, name="evict_one"),
        # all layers of eight rows, whole images held to a thousand positions, prompts kept
        dict(EVICT, name="evict_batch", layers=30, rows=8, kv_heads=8, len_min=1289, len_max=2356, budget_min=1024, budget_max=1024, first_max=312, recent=256,
             page=64, shape_seed=1),
        # long rows, narrow heads, fp32: most positions go
        dict(EVICT, name="evict_long", dtype="f32", layers=2, rows=3, kv_heads=4, head_dim=64, len_min=9000, len_max=16384, budget_min=2000, budget_max=4200,
             first_max=1, recent=1, page=128, shape_seed=2),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case of the ranges above, costing no more than ``shared_trees``, ``mass_chunks`` or ``evict_batch``."""
    kind = rng.choices(["shared", "mass", "evict"], [5, 4, 3])[0]
    seed, page = rng.randrange(1 << 20), rng.choice([16, 16, 32, 48, 64, 128])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (16, 4), (8, 8), (8, 1), (12, 4)])
    f32 = rng.random() < 0.2
    head_dim = rng.choice([64, 80, 128]) if f32 else rng.choice([64, 128, 128])
    base = dict(dtype="f32" if f32 else "bf16", head_dim=head_dim, page=page, shape_seed=seed)
    if kind == "evict":
        length = _log_int(rng, 20, 8000)
        rows = _log_int(rng, 1, 64)
        layers = max(1, min(_log_int(rng, 1, 30), 600000 // (length * rows * kv_heads)))
        budget = _log_int(rng, 10, length)
        return dict(EVICT, **base, layers=layers, rows=min(rows, max(1, 600000 // (length * kv_heads))), kv_heads=kv_heads, len_min=rng.choice([0, length // 2, length]), len_max=length,
                    budget_min=rng.choice([0, budget]), budget_max=budget, first_max=rng.choice([0, 4, budget // 2]), recent=rng.choice([0, 1, budget // 8, budget // 2]))
    if f32:
        heads, kv_heads = 8, rng.choice([8, 2])
    if kind == "mass":
        what = rng.choice(["token", "path", "chunk"])
        prefix = _log_int(rng, 1, 1289 if f32 else 4200)
        case = dict(MASS, **base, heads=heads, kv_heads=kv_heads, prefix_max=prefix, prefix_min=rng.choice([0, prefix // 6, prefix]), first=rng.choice([0, 0, 1, prefix // 3]))
        if rng.random() < 0.25:
            case.update(window=_log_int(rng, 16, 2000), sinks=rng.choice([0, 1, 4, 70]))
        if what == "token":
            return dict(case, rows=_log_int(rng, 1, 64))
        if what == "path":
            return dict(case, rows=_log_int(rng, 1, 32), new_max=_log_int(rng, 1, 60), path=True)
        new = _log_int(rng, 2, 200 if f32 else 1000)
        return dict(case, rows=min(_log_int(rng, 1, 8), max(1, 4000 // new)), new_max=new, new_min=rng.choice([1, max(1, new // 2), new]))
    what = rng.choice(["token", "token", "few", "tree", "chunk"])
    most = _log_int(rng, 16, 1289 if f32 else 8192)
    rows = _log_int(rng, 1, 16 if f32 else 64)
    new, tree = 1, False
    if what == "few":
        new = rng.randint(2, 8)
    elif what == "tree":
        rows, new, tree = min(rows, 16), _log_int(rng, 15, 60 if f32 else 100), True
    elif what == "chunk":
        rows, new = min(rows, 8), _log_int(rng, 9, 100 if f32 else 400)
    if what in ("tree", "chunk"):
        most = min(most, 2048)
    grown = _log_int(rng, 1, 1289)
    return dict(SHARED, **base, rows=rows, groups=rng.randint(1, max(1, rows // 2)), heads=heads, kv_heads=kv_heads, shared_max=most,
                shared_min=rng.choice([0, most // 4, most]), own_max=grown, own_min=rng.choice([0, grown // 4]), new_max=new,
                new_min=max(12, new // 3) if tree else rng.choice([1, new]), tree=tree, depth=rng.randint(3, 10) if tree else 0)


# ---------------------------------------------------------------------------------------------- shapes and inputs

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _shared_shape(case):
    """(group offsets, shared positions of each group, prefix lengths of the rows, their new tokens)."""
    rng = random.Random(case["shape_seed"])
    rows, groups = case["rows"], min(case["groups"], case["rows"])
    cuts = sorted(rng.sample(range(1, rows), groups - 1))
    off = [0, *cuts, rows]
    page = case["page"]
    shared = [rng.randint(case["shared_min"], case["shared_max"]) // page * page for _ in range(groups)]      # whole pages
    prefix = [shared[g] + rng.randint(case["own_min"], case["own_max"]) for g in range(groups) for _ in range(off[g], off[g + 1])]
    return off, shared, prefix, [rng.randint(case["new_min"], case["new_max"]) for _ in range(rows)]


def _mass_shape(case):
    rng = random.Random(case["shape_seed"])
    prefix = [rng.randint(case["prefix_min"], case["prefix_max"]) for _ in range(case["rows"])]
    return prefix, [rng.randint(case["new_min"], case["new_max"]) for _ in range(case["rows"])]


def _evict_shape(case):
    """(lengths, budgets, positions at the front that stay)."""
    rng = random.Random(case["shape_seed"])
    pick = lambda lo, hi: [rng.randint(lo, hi) for _ in range(case["rows"])]  # noqa: E731
    return pick(case["len_min"], case["len_max"]), pick(case["budget_min"], case["budget_max"]), pick(0, case["first_max"])


def _tree(rng, nodes, depth):
    """A drafted tree: one chain of the full depth, the other nodes anywhere above it; parents come first."""
    parent, level = [-1], [0]
    for i in range(1, nodes):
        if i <= min(depth, nodes - 1):
            a = i - 1
        else:
            a = rng.randrange(i)
            while level[a] >= depth:
                a = parent[a]
        parent.append(a)
        level.append(level[a] + 1)
    return parent


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tables(held, seed, same=None):
    """Block tables whose rows hold so many pages, scattered over a pool; `same`: (first row, pages) for every row, whose first pages are that row's.
    What is behind a row's pages is left unset.  Returns the table, the pages of no row, and the pages of the pool."""
    rows = len(held)
    total = sum(held)
    pool = total + total // 8 + 1
    order = np.random.RandomState(seed % (1 << 31)).permutation(pool).astype(np.int32)
    table = np.full((rows, max(max(held), 1)), -1, np.int32)
    at = 0
    for s, n in enumerate(held):
        front = 0
        if same is not None and same[s][0] < s:
            front = same[s][1]
            table[s, :front] = table[same[s][0], :front]
        table[s, front:n] = order[at:at + n - front]
        at += n - front
    return table, order[at:], pool


def prepare(case, seed):
    g = _gen(seed)
    randn = lambda *s, dtype=torch.float32: torch.randn(*s, device="cuda", generator=g, dtype=torch.float32).to(dtype)  # noqa: E731
    st = {"case": case}
    {"shared": _prepare_shared, "mass": _prepare_mass, "evict": _prepare_evict}[case["kind"]](st, case, seed, randn)
    st["ctx"] = _context(case, st)
    if own:
        st["workspace"] = _workspace(st)
    return st


def _prepare_shared(st, case, seed, randn):
    dt, (goff, shared, prefix, new) = _DT[case["dtype"]], _shared_shape(case)
    page, hkv, d, n = case["page"], case["kv_heads"], case["head_dim"], sum(new)
    same = [(goff[g], shared[g] // page) for g in range(len(shared)) for _ in range(goff[g], goff[g + 1])]
    table, _, pool = _tables([-(-p // page) for p in prefix], seed, same)
    off = np.concatenate([[0], np.cumsum(new)])
    st.update(q_off=_ints(off.tolist()), prefix_len=_ints(prefix), block_table=torch.from_numpy(table).cuda(), parent=None, group_off=_ints(goff),
              shared_len=_ints(shared), q=randn(n, case["heads"], d, dtype=dt), k_new=randn(n, hkv, d, dtype=dt), v_new=randn(n, hkv, d, dtype=dt),
              k_pages=randn(pool, hkv, page, d, dtype=dt), v_pages=randn(pool, hkv, page, d, dtype=dt), max_new=max(new), max_prefix=max(prefix), max_shared=max(shared),
              # what a serving program's host knows of its batch: the bounds, for the plain form
              max_rows=max(b - a for a, b in zip(goff, goff[1:])), max_own=max(p - shared[g] for g in range(len(shared)) for p in prefix[goff[g]:goff[g + 1]]),
              max_tokens=max(int(off[b] - off[a]) for a, b in zip(goff, goff[1:])))
    if case["tree"]:
        rng = random.Random(case["shape_seed"] + 1)
        st["parent"] = _ints([a for t in new for a in _tree(rng, t, case["depth"])])
    st.update(out=torch.empty_like(st["q"]), lse=torch.empty(n, case["heads"], device="cuda"))


def _prepare_mass(st, case, seed, randn):
    dt, (prefix, new) = _DT[case["dtype"]], _mass_shape(case)
    page, hkv, d, n, rows = case["page"], case["kv_heads"], case["head_dim"], sum(new), case["rows"]
    length = [p + t for p, t in zip(prefix, new)]
    table, _, pool = _tables([-(-x // page) for x in length], seed)
    off = np.concatenate([[0], np.cumsum(new)])
    st.update(q_off=_ints(off.tolist()), seq_len=_ints(length), block_table=torch.from_numpy(table).cuda(), k_pages=randn(pool, hkv, page, d, dtype=dt), source=None,
              first=_ints([min(case["first"], p) for p in prefix]) if case["first"] else None, max_new=max(new), max_seq=max(length))
    if case["path"]:                  # the kept nodes stand anywhere among all drafted ones, in order; entries behind the last token are unused
        drafted = n + 20 * rows
        kept = np.sort(np.random.RandomState(seed % (1 << 31)).permutation(drafted)[:n])
        st["source"] = _ints([*kept.tolist(), *[-1] * rows])
    else:
        drafted = n
    st["q"] = randn(drafted, case["heads"], d, dtype=dt)
    st["lse"] = torch.full((drafted, case["heads"]), -math.inf, device="cuda")
    at = st["source"][:n].long() if case["path"] else torch.arange(n, device="cuda")
    for lo, hi in _row_runs(length, case["heads"] * max(new)):     # what the attention before it wrote
        score, _ = _mass_scores(st, lo, hi)
        top = score.amax(-1).clamp(min=torch.finfo(torch.float32).min)
        lse = (top + torch.log(torch.exp(score - top[..., None]).sum(-1))).permute(0, 3, 1, 2).reshape(hi - lo, -1, case["heads"])
        there = torch.arange(max(new), device="cuda")[None] < _ints(new[lo:hi])[:, None]
        st["lse"][at[off[lo]:off[hi]]] = lse[there]
    # what earlier tokens left: a few heavy positions, many light ones
    st["mass"] = torch.exp(2 * randn(rows, hkv, max(length) + 13) - 3)


def _row_runs(length, width, most=1 << 28):
    """Runs of rows whose scores fit in so many elements."""
    step = max(1, most // max(1, max(length) * width))
    return [(lo, min(len(length), lo + step)) for lo in range(0, len(length), step)]


def _prepare_evict(st, case, seed, randn):
    dt, (length, budget, first) = _DT[case["dtype"]], _evict_shape(case)
    page, hkv, d, layers, rows = case["page"], case["kv_heads"], case["head_dim"], case["layers"], case["rows"]
    held = [-(-x // page) for x in length]
    table, free, pool = _tables(held, seed)
    pages = np.zeros(pool, np.int32)
    pages[:len(free)] = free
    mass = torch.exp(2 * randn(layers, rows, hkv, max(length) + 5) - 3)
    mass *= randn(layers, rows, hkv, max(length) + 5) > -1.3            # a tenth of them nothing ever attended: equal weights
    k = randn(1, pool, hkv, page, d, dtype=dt).expand(layers, pool, hkv, page, d).contiguous()
    st.update(seq_len=_ints(length), budget=_ints(budget), n_first=_ints(first), block_table=torch.from_numpy(table).cuda(), mass=mass,
              mass_out=torch.zeros_like(mass), free_pages=torch.from_numpy(pages).cuda(), free_count=_ints([len(free)]), k_pages=k, v_pages=-k,
              seq_len_out=torch.empty(rows, dtype=torch.int32, device="cuda"), free_count_out=torch.empty(1, dtype=torch.int32, device="cuda"),
              dropped=torch.empty(rows, dtype=torch.int32, device="cuda"), max_seq=max(length))


def _context(case, st):
    """The handle that a serving program keeps."""
    if not own:
        return None
    from paper_2605_07230_amd import binding
    rows = case["rows"]
    n = st["q"].shape[0] if "q" in st else rows
    if st.get("source") is not None:
        n = max(n, st["source"].numel())
    return binding.Context(max_rows=rows, max_nodes_total=n, max_nodes_per_tree=min(1024, max(1, st.get("max_new", 1))),
                           max_prefix=max(1, st.get("max_prefix", st.get("max_seq", 1))), n_heads=case.get("heads", case["kv_heads"]), head_dim=case["head_dim"],
                           hidden=64, vocab=64)


def _workspace(st):
    """Scratch of a call, which such a program keeps too."""
    from paper_2605_07230_amd import binding
    if st["case"]["kind"] == "mass":
        return None
    if st["case"]["kind"] == "shared":
        size = binding.paged_attn_shared_workspace(st["ctx"], **_shared_args(st))
    else:
        size = binding.paged_evict_workspace(st["ctx"], **_evict_args(st))
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    kind = st["case"]["kind"]
    if own:
        return _RUN_OWN[kind](st)
    return _RUN_PLAIN[kind](st)


def _shared_args(st):
    return dict(q_off=st["q_off"], parent=st["parent"], prefix_len=st["prefix_len"], block_table=st["block_table"], q=st["q"], k_new=st["k_new"],
                v_new=st["v_new"], k_pages=st["k_pages"], v_pages=st["v_pages"], out=st["out"], lse=st["lse"], max_new=st["max_new"],
                max_prefix_len=st["max_prefix"], group_off=st["group_off"], shared_len=st["shared_len"], max_shared_len=st["max_shared"])


def _own_shared(st):
    from paper_2605_07230_amd import binding
    binding.paged_attn_shared(st["ctx"], workspace=st["workspace"], **_shared_args(st))
    return {"out": st["out"], "lse": st["lse"]}


def _own_mass(st):
    from paper_2605_07230_amd import binding
    c = st["case"]
    binding.paged_mass(st["ctx"], q_off=st["q_off"], seq_len=st["seq_len"], block_table=st["block_table"], q=st["q"], lse=st["lse"], k_pages=st["k_pages"],
                       mass=st["mass"], source=st["source"], first=st["first"], window=c["window"], n_sink=c["sinks"], max_new=st["max_new"],
                       max_seq_len=st["max_seq"])
    return {"mass": st["mass"]}


def _evict_args(st):
    return dict(seq_len=st["seq_len"], budget=st["budget"], n_first=st["n_first"], n_recent=st["case"]["recent"], block_table=st["block_table"],
                k_pages=st["k_pages"], v_pages=st["v_pages"], mass=st["mass"], mass_out=st["mass_out"], free_pages=st["free_pages"],
                free_count=st["free_count"], seq_len_out=st["seq_len_out"], free_count_out=st["free_count_out"], dropped=st["dropped"], max_seq_len=st["max_seq"])


def _own_evict(st):
    from paper_2605_07230_amd import binding
    binding.paged_evict(st["ctx"], workspace=st["workspace"], **_evict_args(st))
    return {k: st[k] for k in ("k_pages", "v_pages", "mass_out", "free_pages", "seq_len_out", "free_count_out", "dropped")}


def _squared(m):
    return torch.clamp(m @ m, max=1.0)


def _softmax_part(score, v, lead):
    """(maximum, sum, weighted values) of scores [.., queries, keys] whose queries stand in `lead` dimensions."""
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    weight = torch.exp(score - top)
    return top[..., 0], weight.sum(-1), (weight.reshape(*v.shape[:2], -1, v.shape[2]) @ v).reshape(*lead, v.shape[3])


def _plain_shared(st):
    c = st["case"]
    page, hkv, heads, d, rows = c["page"], c["kv_heads"], c["heads"], c["head_dim"], c["rows"]
    off, goff, shared, prefix = (st[k].long() for k in ("q_off", "group_off", "shared_len", "prefix_len"))
    t, n, G, cuda = st["max_new"], st["q"].shape[0], heads // hkv, "cuda"
    groups, ms, mo = shared.numel(), max(st["max_shared"], 1), max(st["max_own"], 1)
    scale = 1.0 / math.sqrt(d)
    table = st["block_table"].long()
    table = torch.cat([table, table.new_zeros(rows, 1)], 1)
    # ---- the shared keys, once for a group
    first, last = off[goff[:-1]], off[goff[1:]]
    i = torch.arange(st["max_tokens"], device=cuda)
    in_group = i[None] < (last - first)[:, None]
    at = torch.where(in_group, first[:, None] + i[None], 0)
    pos = torch.arange(ms, device=cuda)
    held = pos[None] < shared[:, None]
    entry = torch.where(held, table[goff[:-1]][:, pos // page % table.shape[1]], 0)
    k, v = (st[x][entry, :, pos % page].float().transpose(1, 2) for x in ("k_pages", "v_pages"))                # [groups, hkv, ms, d]
    q = st["q"][at].float().view(groups, -1, hkv, G, d).permute(0, 2, 3, 1, 4)                                  # [groups, hkv, G, tokens, d]
    score = (q.reshape(groups, hkv, -1, d) @ k.transpose(2, 3) * scale).masked_fill(~held[:, None, None], -math.inf)
    m0, l0, o0 = _softmax_part(score.view(groups, hkv, G, -1, ms), v, (groups, hkv, G, at.shape[1]))
    pick = in_group.reshape(-1).nonzero()[:, 0]
    m0, l0 = (x.permute(0, 3, 1, 2).reshape(-1, heads)[pick] for x in (m0, l0))
    o0 = o0.permute(0, 3, 1, 2, 4).reshape(-1, heads, d)[pick]
    # ---- the rows' own keys and new tokens
    row_shared = shared.repeat_interleave(goff[1:] - goff[:-1], output_size=rows)
    i = torch.arange(t, device=cuda)
    there = i[None] < (off[1:] - off[:-1])[:, None]
    at = torch.where(there, off[:-1, None] + i[None], 0)
    pos = torch.arange(mo, device=cuda)[None] + row_shared[:, None]
    cached = pos < prefix[:, None]
    entry = torch.where(cached, table.gather(1, (pos // page).clamp(max=table.shape[1] - 1)), 0)
    k, v = (torch.cat([st[x][entry, :, pos % page].float(), st[y][at].float()], 1).transpose(1, 2) for x, y in (("k_pages", "k_new"), ("v_pages", "v_new")))
    if st["parent"] is None:
        sees = (i[None, None] <= i[None, :, None]).expand(rows, t, t)
    else:
        parent = torch.where(there, st["parent"].long()[at], -1)
        reach = (parent[..., None] == i[None, None]).float() + torch.eye(t, device=cuda)
        sees = _squared(_squared(_squared(_squared(reach)))) > 0                     # depths of up to 16
    mask = torch.cat([cached[:, None].expand(rows, t, mo), sees & there[:, None]], 2)
    q = st["q"][at].float().view(rows, t, hkv, G, d).permute(0, 2, 3, 1, 4)
    score = (q.reshape(rows, hkv, -1, d) @ k.transpose(2, 3) * scale).view(rows, hkv, G, t, mo + t).masked_fill(~mask[:, None, None], -math.inf)
    m1, l1, o1 = _softmax_part(score, v, (rows, hkv, G, t))
    pick = there.reshape(-1).nonzero()[:, 0]
    m1, l1 = (x.permute(0, 3, 1, 2).reshape(-1, heads)[pick] for x in (m1, l1))
    o1 = o1.permute(0, 3, 1, 2, 4).reshape(-1, heads, d)[pick]
    # ---- joined
    m = torch.maximum(m0, m1)
    f0, f1 = torch.exp(m0 - m), torch.exp(m1 - m)
    total = f0 * l0 + f1 * l1
    out = (f0[..., None] * o0 + f1[..., None] * o1) / total[..., None]
    return {"out": out.to(st["q"].dtype), "lse": m + torch.log(total)}


def _mass_scores(st, lo, hi):
    """Scores of rows lo .. hi - 1, [rows, hkv, G, tokens, keys] in 32 bits, -inf where a token does not attend, and the tokens that exist."""
    c = st["case"]
    page, hkv, heads, d = c["page"], c["kv_heads"], c["heads"], c["head_dim"]
    off, length = st["q_off"].long(), st["seq_len"].long()[lo:hi]
    t, G, rows, keys = st["max_new"], heads // hkv, hi - lo, st["max_seq"]
    count = off[lo + 1:hi + 1] - off[lo:hi]
    i, pos = torch.arange(t, device="cuda"), torch.arange(keys, device="cuda")
    there = i[None] < count[:, None]
    at = torch.where(there, off[lo:hi, None] + i[None], 0)
    if st["source"] is not None:
        at = st["source"].long()[at]
    cached = pos[None] < length[:, None]
    entry = torch.where(cached, st["block_table"].long()[lo:hi].repeat_interleave(page, 1)[:, :keys], 0)
    k = st["k_pages"][entry, :, pos % page].float().permute(0, 2, 3, 1)                                         # [rows, hkv, d, keys]
    q = st["q"][at].float().view(rows, t, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(rows, hkv, -1, d)
    x = (length - count)[:, None] + i[None]
    mask = (pos[None, None] <= x[:, :, None]) & there[:, :, None]
    if c["window"]:
        mask = mask & ((x[:, :, None] - pos[None, None] < c["window"]) | (pos[None, None] < c["sinks"]))
    score = (q @ k).mul_(1.0 / math.sqrt(d)).view(rows, hkv, G, t, keys).masked_fill_(~mask[:, None, None], -math.inf)
    return score, at


def _plain_mass(st):
    c = st["case"]
    rows, keys, hkv = c["rows"], st["max_seq"], c["kv_heads"]
    score, at = _mass_scores(st, 0, rows)
    lse = st["lse"][at].view(rows, -1, hkv, c["heads"] // hkv).permute(0, 2, 3, 1)[..., None]
    new = torch.exp(score.sub_(lse)).sum((2, 3))                                                               # [rows, hkv, keys]
    length = st["seq_len"].long()
    pos = torch.arange(keys, device="cuda")
    before = length - (st["q_off"][1:] - st["q_off"][:-1]).long()
    old = st["mass"][:, :, :keys]
    seen = (pos[None] < length[:, None]) & (pos[None] >= (st["first"].long() if st["first"] is not None else torch.zeros_like(length))[:, None])
    st["mass"][:, :, :keys] = torch.where(seen[:, None], torch.where((pos[None] < before[:, None])[:, None], old + new, new), old)
    return {"mass": st["mass"]}


def _plain_evict(st):
    c = st["case"]
    page, rows, keys, recent = c["page"], c["rows"], st["max_seq"], c["recent"]
    length, budget, table = st["seq_len"].long(), st["budget"].long(), st["block_table"].long()
    first = torch.minimum(st["n_first"].long(), length)
    tail = torch.minimum(torch.full_like(length, recent), length - first)
    after = torch.maximum(torch.minimum(budget, length), first + tail)
    middle = after - tail
    pos = torch.arange(keys, device="cuda")
    per_row = lambda x: x[None, :, None, None]  # noqa: E731
    free = (pos >= per_row(first)) & (pos < per_row(length - tail))                      # those that the weight decides on
    mass = torch.where(free, st["mass"][..., :keys], -1.0)
    order = torch.sort(mass, dim=-1, descending=True, stable=True).indices               # of equal ones the first
    rank = torch.empty_like(order).scatter_(-1, order, pos.expand_as(order))
    kept = free & (rank < per_row(middle - first))
    hole = free & ~kept & (pos < per_row(middle))
    fill = kept & (pos >= per_row(middle))
    # the j-th hole gets the j-th kept position behind the middle; the last ones move down in order
    source = pos.expand_as(order).clone()
    source[hole] = pos.expand_as(order)[fill]
    source = torch.where((pos >= per_row(middle)) & (pos < per_row(after)), pos + per_row(length - after), source)
    st["mass_out"][..., :keys] = torch.where(pos < per_row(after), st["mass"][..., :keys].gather(-1, source.clamp(max=keys - 1)), st["mass_out"][..., :keys])
    moved = ((source != pos) & (pos < per_row(after))).nonzero()
    layer, row, head, to = moved.unbind(1)
    come = source[layer, row, head, to]
    where = lambda p: (layer, table[row, p // page], head, p % page)  # noqa: E731
    st["k_pages"][where(to)] = st["k_pages"][where(come)]
    st["v_pages"][where(to)] = st["v_pages"][where(come)]
    left, held = (after + page - 1) // page, (length + page - 1) // page
    e = torch.arange(table.shape[1], device="cuda")
    back = st["block_table"][(e >= left[:, None]) & (e < held[:, None])]                # row by row
    at = st["free_count"].long() + torch.arange(back.numel(), device="cuda")
    st["free_pages"][at] = back
    return {"k_pages": st["k_pages"], "v_pages": st["v_pages"], "mass_out": st["mass_out"], "free_pages": st["free_pages"], "seq_len_out": after.int(),
            "free_count_out": (st["free_count"] + back.numel()).int(), "dropped": (length - after).int()}


_RUN_OWN = {"shared": _own_shared, "mass": _own_mass, "evict": _own_evict}
_RUN_PLAIN = {"shared": _plain_shared, "mass": _plain_mass, "evict": _plain_evict}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    d, hkv = case["head_dim"], case["kv_heads"]
    if case["kind"] == "evict":
        moved = entries = weights = 0
        for length, budget, first in zip(*_evict_shape(case)):
            first = min(first, length)
            recent = min(case["recent"], length - first)
            after = max(min(budget, length), first + recent)
            gone = length - after
            # positions of the middle that fall among the heaviest by chance stay where they are
            free = length - recent - first
            moved += (after - recent - first) * gone / max(free, 1) + (recent if gone else 0)
            entries += -(-length // case["page"]) - -(-after // case["page"])
            weights += length + after
        heads = case["layers"] * hkv
        return {"bytes": int(heads * (4 * moved * d * size + 4 * weights) + 8 * entries + 20 * case["rows"]), "flops": heads * weights}
    if case["kind"] == "mass":
        prefix, new = _mass_shape(case)
        w, sinks = case["window"], case["sinks"]
        keys = pairs = 0
        for p, t in zip(prefix, new):
            first = min(case["first"], p)
            for x in range(p, p + t):
                seen = x + 1
                pairs += max(0, min(seen, w + min(sinks, max(0, seen - w))) if w else seen - first)
            keys += t + (min(p - first, w - 1 + sinks) if w else p - first)
        n = sum(new)
        return {"bytes": keys * hkv * (d * size + 8) + n * case["heads"] * (d * size + 4), "flops": 2 * d * case["heads"] * pairs}
    goff, shared, prefix, new = _shared_shape(case)
    keys, pairs = sum(shared), 0
    rng = random.Random(case["shape_seed"] + 1)
    for g, (lo, hi) in enumerate(zip(goff, goff[1:])):
        for s in range(lo, hi):
            level = list(range(new[s]))
            if case["tree"]:
                level = [0]
                for a in _tree(rng, new[s], case["depth"])[1:]:
                    level.append(level[a] + 1)
            pairs += sum(prefix[s] + x + 1 for x in level)
            keys += prefix[s] - shared[g] + new[s]
    n = sum(new)
    return {"bytes": 2 * keys * hkv * d * size + 2 * n * case["heads"] * d * size + 4 * n * case["heads"] + 4 * keys // case["page"],
            "flops": 4 * d * case["heads"] * pairs}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits, row by row

def exact(case, seed):
    st = prepare(case, seed)
    return {"shared": _exact_shared, "mass": _exact_mass, "evict": _exact_evict}[case["kind"]](st, case)


def _exact_shared(st, case):
    off, prefix, page = st["q_off"].tolist(), st["prefix_len"].tolist(), case["page"]
    table = st["block_table"].cpu().numpy()
    parent = None if st["parent"] is None else st["parent"].cpu().numpy()
    group = case["heads"] // case["kv_heads"]
    out, lse = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for s in range(case["rows"]):
        lo, hi, p = off[s], off[s + 1], prefix[s]
        where = np.arange(p)
        pg, inside = torch.from_numpy(table[s, where // page].astype(np.int64)).cuda(), torch.from_numpy(where % page).cuda()
        sees = np.zeros((hi - lo, hi - lo), bool)
        for i in range(hi - lo):
            if parent is None:
                sees[i, :i + 1] = True
            else:
                a = i
                while a >= 0:
                    sees[i, a] = True
                    a = int(parent[lo + a])
        sees = torch.from_numpy(np.concatenate([np.ones((hi - lo, p), bool), sees], 1)).cuda()
        for h in range(case["kv_heads"]):
            key = torch.cat([st["k_pages"][pg, h, inside], st["k_new"][lo:hi, h]]).double()
            val = torch.cat([st["v_pages"][pg, h, inside], st["v_new"][lo:hi, h]]).double()
            q = st["q"][lo:hi, h * group:(h + 1) * group].double()
            z = (q.reshape(-1, q.shape[-1]) @ key.T / math.sqrt(case["head_dim"])).view(hi - lo, group, -1).masked_fill(~sees[:, None], -math.inf)
            lse[lo:hi, h * group:(h + 1) * group] = torch.logsumexp(z, 2)
            out[lo:hi, h * group:(h + 1) * group] = (torch.softmax(z, 2).view((hi - lo) * group, -1) @ val).view(hi - lo, group, -1)
    return {"out": out, "lse": lse}


def _exact_mass(st, case):
    off, length, page = st["q_off"].tolist(), st["seq_len"].tolist(), case["page"]
    table = st["block_table"].cpu().numpy()
    group, mass = case["heads"] // case["kv_heads"], st["mass"].double()
    for s in range(case["rows"]):
        n, where = off[s + 1] - off[s], np.arange(length[s])
        pg, inside = torch.from_numpy(table[s, where // page].astype(np.int64)).cuda(), torch.from_numpy(where % page).cuda()
        tokens = torch.arange(off[s], off[s + 1], device="cuda")
        if st["source"] is not None:
            tokens = st["source"][tokens].long()
        x = torch.arange(length[s] - n, length[s], device="cuda")
        y = torch.from_numpy(where).cuda()
        sees = y[None] <= x[:, None]
        if case["window"]:
            sees &= (x[:, None] - y[None] < case["window"]) | (y[None] < case["sinks"])
        first = 0 if st["first"] is None else int(st["first"][s])
        for h in range(case["kv_heads"]):
            key = st["k_pages"][pg, h, inside].double()
            q, top = st["q"][tokens, h * group:(h + 1) * group].double(), st["lse"][tokens, h * group:(h + 1) * group].double()
            z = (q.reshape(-1, q.shape[-1]) @ key.T / math.sqrt(case["head_dim"])).view(n, group, -1) - top[..., None]
            got = torch.where(sees[:, None], torch.exp(z), 0.0).sum((0, 1))
            got[:length[s] - n] += mass[s, h, :length[s] - n]
            mass[s, h, first:length[s]] = got[first:]
    return {"mass": mass}


def _exact_evict(st, case):
    """Weights are moved, not computed: the ones that stand in each place, by sorting (weight, position) on the host."""
    length, budget, first = _evict_shape(case)
    if sum(length) * case["layers"] * case["kv_heads"] > 1 << 20:
        return None
    mass, out = st["mass"].double().cpu().numpy(), st["mass_out"].double().cpu().numpy()
    for s, (n, b, f) in enumerate(zip(length, budget, first)):
        f = min(f, n)
        r = min(case["recent"], n - f)
        after = max(min(b, n), f + r)
        for layer in range(case["layers"]):
            for h in range(case["kv_heads"]):
                w = mass[layer, s, h]
                best = sorted(range(f, n - r), key=lambda y: (-w[y], y))[:after - r - f]
                keep = set(best)
                come = sorted(y for y in best if y >= after - r)
                place = [*range(f), *(y if y in keep else -1 for y in range(f, after - r))]
                for i, y in enumerate(place):
                    if y < 0:
                        place[i] = come.pop(0)
                out[layer, s, h, :after] = w[place + list(range(n - r, n))]
    return {"k_pages": None, "v_pages": None, "mass_out": torch.from_numpy(out), "free_pages": None, "seq_len_out": None, "free_count_out": None, "dropped": None}
