"""Serving operators around the verification step: what they are timed on, how inputs are made, and one pass through each.

``attn``    attention of new tokens (a prompt's chunk, a single token, a drafted tree) over a cache in pages
``append``  the copy of new tokens' keys and values into the pages of every decoder layer
``slots``   pages for requests that grow: block tables, slot maps, positions
``sample``  tokens drawn from rows of logits with each row's own temperature, top-k, top-p and min-p

Where ``own`` is false a pass is written in elementary torch operations, in 32 bits (sampling in 64: a draw has to land on the same
token); where it is true it is the call of ``paper_2605_07230_amd.binding`` that a serving program makes.  Sizes are the
repository's own configurations (``workloads.make_config``, ``bench.py``, ``perf/cases.py``) and the ranges between them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

ATTN = dict(kind="attn", dtype="bf16", rows=2, heads=32, kv_heads=32, head_dim=128, prefix_min=312, prefix_max=312, new_min=1, new_max=1,
            page=16, window=0, sinks=0, tree=False, depth=0, shape_seed=0)
APPEND = dict(kind="append", dtype="bf16", layers=30, rows=16, kv_heads=32, head_dim=128, new_min=1, new_max=1, prefix_max=600, page=16, shape_seed=0)
SLOTS = dict(kind="slots", rows=16, prefix_min=100, prefix_max=600, new_min=1, new_max=1, page=16, path=False, depth=0, shape_seed=0)
SAMPLE = dict(kind="sample", dtype="f32", rows=1, vocab=16384, sigma=2.0, temperature="1", top_k="2000", top_p="1", min_p="0", shape_seed=0)


def listed():
    return [
        # plain decoding of one user and the guidance row, 312 tokens in the cache: latency of a single token
        dict(ATTN, name="attn_token"),
        # plain decoding of a full batch: 64 requests anywhere in their images, grouped heads; the cache streams
        dict(ATTN, name="attn_token_batch", rows=64, kv_heads=8, prefix_min=90, prefix_max=4200, page=32, shape_seed=1),
        # prompts that arrive in chunks, ragged, some with chunks before them in the cache: products bound it
        dict(ATTN, name="attn_chunks", rows=8, kv_heads=8, prefix_min=0, prefix_max=2000, new_min=500, new_max=1000, page=64, shape_seed=2),
        # a long chunk under a sliding window with a few first tokens kept, narrow heads
        dict(ATTN, name="attn_window", rows=2, heads=16, kv_heads=4, head_dim=64, prefix_min=4000, prefix_max=4200, new_min=1800, new_max=2000,
             page=16, window=1024, sinks=4, shape_seed=3),
        # verification of 256-node trees at 4200 keys for eight rows, as bench.py's headline does it, with the prefixes in pages
        dict(ATTN, name="attn_trees", rows=8, prefix_min=4200, prefix_max=4200, new_min=256, new_max=256, page=16, tree=True, depth=10, shape_seed=4),
        # the fp32 configuration: fifteen new tokens behind 256
        dict(ATTN, name="attn_f32", dtype="f32", rows=1, heads=8, kv_heads=8, head_dim=64, prefix_min=256, prefix_max=256, new_min=15, new_max=15,
             page=16, shape_seed=5),
        # one new token of each of 16 rows, all layers
        dict(APPEND, name="append_tokens"),
        # a batch of prompts, all layers
        dict(APPEND, name="append_prompts", rows=8, kv_heads=8, new_min=200, new_max=312, prefix_max=0, page=64, shape_seed=1),
        # what a verification step keeps: eight prompts with their guidance rows, accepted paths of up to ten nodes
        dict(SLOTS, name="slots_path", path=True, depth=10),
        # a full batch of prompts admitted at once
        dict(SLOTS, name="slots_prompts", rows=256, prefix_min=0, prefix_max=2000, new_min=1, new_max=1289, shape_seed=1),
        # one row with the paper's top-k, image vocabulary
        dict(SAMPLE, name="sample_one"),
        # a full batch of the large vocabulary, every request with parameters of its own, greedy ones among them
        dict(SAMPLE, name="sample_batch", rows=256, vocab=65536, temperature="0,0.7,1,1.3", top_k="0,50,2000", top_p="1,0.9,0.95", min_p="0,0,0.05",
             shape_seed=1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """One more case of the ranges above, costing no more than ``attn_trees`` or ``append_prompts``."""
    kind = rng.choices(["attn", "append", "slots", "sample"], [6, 1, 1, 3])[0]
    seed, page = rng.randrange(1 << 20), rng.choice([16, 16, 32, 48, 64, 128])
    if kind == "append":
        rows, new = _log_int(rng, 1, 64), _log_int(rng, 1, 312)
        new = max(1, min(new, 2000 // rows))
        return dict(APPEND, dtype=rng.choice(["bf16", "bf16", "f32"]), layers=rng.randint(1, 30), rows=rows, kv_heads=rng.choice([1, 4, 8]),
                    head_dim=rng.choice([64, 128]), new_min=rng.choice([1, new]), new_max=new, prefix_max=_log_int(rng, 1, 600), page=page, shape_seed=seed)
    if kind == "slots":
        path = rng.random() < 0.5
        new = _log_int(rng, 1, 1289)
        return dict(SLOTS, rows=2 * _log_int(rng, 1, 128), prefix_min=0, prefix_max=_log_int(rng, 1, 4200), new_min=rng.choice([0, 1, new]), new_max=new,
                    page=page, path=path, depth=rng.randint(1, 60) if path else 0, shape_seed=seed)
    if kind == "sample":
        pick = lambda *some: rng.choice(some)  # noqa: E731
        return dict(SAMPLE, dtype=pick("f32", "f32", "bf16"), rows=_log_int(rng, 1, 256), vocab=rng.choice([4096, 16384, 33088, 65536, rng.randint(500, 65536)]),
                    sigma=pick(1.0, 2.0, 4.0), temperature=pick("1", "0.7", "0,0.5,1,1.5"), top_k=pick("0", "2000", "0,1,40,300,2000"),
                    top_p=pick("1", "0.9", "1,0.5,0.8,0.99"), min_p=pick("0", "0.02", "0,0.001,0.1"), shape_seed=seed)
    head_dim = rng.choice([64, 128, 128])
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (16, 4), (8, 8), (8, 1), (12, 4)])
    what = rng.choice(["token", "token", "chunk", "chunk", "tree", "f32"])
    if what == "f32":
        new = _log_int(rng, 1, 200)
        return dict(ATTN, dtype="f32", rows=_log_int(rng, 1, 8), heads=8, kv_heads=rng.choice([8, 2]), head_dim=rng.choice([64, 80, 128]), prefix_min=0,
                    prefix_max=_log_int(rng, 1, 1289), new_min=1, new_max=new, page=page, window=rng.choice([0, 0, 100]), sinks=rng.choice([0, 3]), shape_seed=seed)
    prefix = _log_int(rng, 16, 4200)
    out = dict(ATTN, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, prefix_max=prefix, prefix_min=rng.choice([0, prefix // 6, prefix]), shape_seed=seed)
    if what == "tree":
        nodes = _log_int(rng, 15, 256)
        return dict(out, rows=_log_int(rng, 1, 8), new_max=nodes, new_min=rng.choice([max(12, nodes // 3), nodes]), tree=True, depth=rng.randint(3, 10))
    if rng.random() < 0.3:
        out.update(window=_log_int(rng, 16, 2000), sinks=rng.choice([0, 1, 4, 70]))
    if what == "token":
        return dict(out, rows=_log_int(rng, 1, 64))
    new = _log_int(rng, 2, 1000)
    return dict(out, rows=min(_log_int(rng, 1, 8), max(1, 4000 // new)), new_max=new, new_min=rng.choice([1, max(1, new // 2), new]))


# ---------------------------------------------------------------------------------------------- shapes and inputs

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _lengths(case):
    """(prefix lengths, new tokens) of a case's rows."""
    rng = random.Random(case["shape_seed"])
    prefix = [rng.randint(case.get("prefix_min", 0), case["prefix_max"]) for _ in range(case["rows"])]
    if case.get("path"):
        kept = [rng.randint(0, case["depth"]) for _ in range(case["rows"] // 2)]      # a prompt's two rows keep the same path
        return [prefix[s // 2] for s in range(case["rows"])], [1 + kept[s // 2] for s in range(case["rows"])]
    return prefix, [rng.randint(case["new_min"], case["new_max"]) for _ in range(case["rows"])]


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


def _tables(pages_held, width, seed):
    """Block tables whose rows hold so many pages, scattered over a pool; what is behind them is left unset."""
    rows, total = len(pages_held), sum(pages_held)
    pool = total + total // 4 + 1
    order = np.random.RandomState(seed % (1 << 31)).permutation(pool).astype(np.int32)
    table = np.full((rows, max(width, 1)), -1, np.int32)
    at = 0
    for s, n in enumerate(pages_held):
        table[s, :n] = order[at:at + n]
        at += n
    return table, order[at:], pool


def prepare(case, seed):
    g = _gen(seed)
    randn = lambda *s, dtype=torch.float32: torch.randn(*s, device="cuda", generator=g, dtype=torch.float32).to(dtype)  # noqa: E731
    st = {"case": case}
    if case["kind"] == "sample":
        _prepare_sample(st, case, g, seed)
    elif case["kind"] == "slots":
        _prepare_slots(st, case, seed)
    else:
        dt, (prefix, new) = _DT[case["dtype"]], _lengths(case)
        page, hkv, d, n = case["page"], case["kv_heads"], case["head_dim"], sum(new)
        append = case["kind"] == "append"
        ends = [p + t if append else p for p, t in zip(prefix, new)]
        held = [-(-e // page) for e in ends]
        table, _, pool = _tables(held, max(held), seed)
        if append:
            slots = [int(table[s, x // page]) * page + x % page for s in range(len(new)) for x in range(prefix[s], ends[s])]
            st.update(slot_map=_ints(slots), k_new=randn(case["layers"], n, hkv, d, dtype=dt), v_new=randn(case["layers"], n, hkv, d, dtype=dt),
                      k_pages=randn(1, 1, hkv, page, d, dtype=dt).expand(case["layers"], pool, hkv, page, d).contiguous())
            st["v_pages"] = -st["k_pages"]
        else:
            off = np.concatenate([[0], np.cumsum(new)])
            st.update(q_off=_ints(off.tolist()), prefix_len=_ints(prefix), block_table=torch.from_numpy(table).cuda(), parent=None,
                      q=randn(n, case["heads"], d, dtype=dt), k_new=randn(n, hkv, d, dtype=dt), v_new=randn(n, hkv, d, dtype=dt),
                      k_pages=randn(pool, hkv, page, d, dtype=dt), v_pages=randn(pool, hkv, page, d, dtype=dt), max_new=max(new), max_prefix=max(prefix))
            if case["tree"]:
                rng = random.Random(case["shape_seed"] + 1)
                st["parent"] = _ints([a for t in new for a in _tree(rng, t, case["depth"])])
            st.update(out=torch.empty_like(st["q"]), lse=torch.empty(n, case["heads"], device="cuda"))
    st["ctx"] = _context(case, st)
    return st


def _prepare_sample(st, case, g, seed):
    rows, vocab = case["rows"], case["vocab"]
    rng = random.Random(case["shape_seed"])
    some = lambda key, kind: [kind(rng.choice(case[key].split(","))) for _ in range(rows)]  # noqa: E731
    st.update(logits=(case["sigma"] * torch.randn(rows, vocab, device="cuda", generator=g)).to(_DT[case["dtype"]]),
              temperature=torch.tensor(some("temperature", float), device="cuda"), top_k=_ints(some("top_k", int)),
              top_p=torch.tensor(some("top_p", float), device="cuda"), min_p=torch.tensor(some("min_p", float), device="cuda"),
              u=torch.rand(rows, device="cuda", generator=g), token=torch.empty(rows, dtype=torch.int32, device="cuda"),
              prob=torch.empty(rows, device="cuda"))


def _prepare_slots(st, case, seed):
    prefix, new = _lengths(case)
    page, rows = case["page"], case["rows"]
    held = [-(-p // page) for p in prefix]
    need = sum(-(-(p + t) // page) for p, t in zip(prefix, new)) - sum(held)
    width = -(-max(p + t for p, t in zip(prefix, new)) // page)
    table, free, pool = _tables([h + -(-need // rows) for h in held], width + -(-need // rows), seed)
    for s, h in enumerate(held):                      # the pages that the rows ask for lie in the list of free ones, on top of spare ones
        free = np.concatenate([free, table[s, h:][table[s, h:] >= 0]])
        table[s, h:] = -1
    tokens = sum(new)
    st.update(seq_len=_ints(prefix), block_table=torch.from_numpy(table).cuda(), free_pages=torch.from_numpy(free).cuda(), free_count=_ints([len(free)]),
              n_pages=pool, new_len=None, row_prompt=None, accept_len=None, path_nodes=None, node_off=None, n_nodes=0)
    if case["path"]:
        depth, nodes = case["depth"], case["depth"] + 20
        rng = random.Random(seed)
        paths = []
        for s in range(0, rows, 2):
            path = sorted(rng.sample(range(1, nodes), new[s] - 1))
            paths.append(path + [-1] * (depth - len(path)))
        st.update(row_prompt=_ints([s // 2 for s in range(rows)]), accept_len=_ints([new[s] - 1 for s in range(0, rows, 2)]), path_nodes=_ints(paths),
                  node_off=_ints([nodes * s for s in range(rows + 1)]), n_nodes=nodes * rows)
        tokens = rows * (depth + 1)
    else:
        st["new_len"] = _ints(new)
    one = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    st.update(q_off=one(rows + 1), slot_map=one(tokens), position=one(tokens), source=one(tokens), seq_len_out=one(rows), free_count_out=one(1))


def _context(case, st):
    """The handle that a serving program keeps."""
    if not own:
        return None
    from paper_2605_07230_amd import binding
    rows = case["rows"]
    n = st["q"].shape[0] if "q" in st else st["slot_map"].numel() if "slot_map" in st else rows
    return binding.Context(max_rows=rows, max_nodes_total=max(n, st.get("n_nodes", 0)), max_nodes_per_tree=min(1024, max(1, st.get("max_new", 1))),
                           max_prefix=max(1, st.get("max_prefix", 1)), n_heads=case.get("heads", 1), head_dim=case.get("head_dim", 64), hidden=64,
                           vocab=case.get("vocab", 64))


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    kind = st["case"]["kind"]
    if own:
        return _RUN_OWN[kind](st)
    return _RUN_PLAIN[kind](st)


def _own_attn(st):
    from paper_2605_07230_amd import binding
    c = st["case"]
    binding.paged_attn(st["ctx"], q_off=st["q_off"], parent=st["parent"], prefix_len=st["prefix_len"], block_table=st["block_table"], q=st["q"],
                       k_new=st["k_new"], v_new=st["v_new"], k_pages=st["k_pages"], v_pages=st["v_pages"], out=st["out"], lse=st["lse"],
                       window=c["window"], n_sink=c["sinks"], max_new=st["max_new"], max_prefix_len=st["max_prefix"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_append(st):
    from paper_2605_07230_amd import binding
    binding.paged_append(st["ctx"], k_new=st["k_new"], v_new=st["v_new"], slot_map=st["slot_map"], k_pages=st["k_pages"], v_pages=st["v_pages"])
    return {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _own_slots(st):
    from paper_2605_07230_amd import binding
    binding.paged_slots(st["ctx"], seq_len=st["seq_len"], new_len=st["new_len"], block_table=st["block_table"], free_pages=st["free_pages"],
                        free_count=st["free_count"], page_size=st["case"]["page"], n_pages=st["n_pages"], q_off=st["q_off"], slot_map=st["slot_map"],
                        position=st["position"], source=st["source"], seq_len_out=st["seq_len_out"], free_count_out=st["free_count_out"],
                        row_prompt=st["row_prompt"], accept_len=st["accept_len"], path_nodes=st["path_nodes"], node_off=st["node_off"],
                        n_nodes_total=st["n_nodes"])
    return {k: st[k] for k in ("q_off", "slot_map", "position", "source", "seq_len_out", "free_count_out", "block_table")}


def _own_sample(st):
    from paper_2605_07230_amd import binding
    binding.sample_tokens(st["ctx"], logits=st["logits"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                          u=st["u"], token=st["token"], prob=st["prob"])
    return {"token": st["token"], "prob": st["prob"]}


def _squared(m):
    return torch.clamp(m @ m, max=1.0)


def _plain_attn(st):
    c = st["case"]
    off, prefix, page = st["q_off"].long(), st["prefix_len"].long(), c["page"]
    n, heads, d = st["q"].shape
    rows, hkv, t, pm = c["rows"], c["kv_heads"], st["max_new"], st["max_prefix"]
    count = off[1:] - off[:-1]
    i = torch.arange(t, device="cuda")
    there = i[None] < count[:, None]                                            # [rows, t]
    at = torch.where(there, off[:-1, None] + i[None], 0)
    # keys: the prefix through the table, then the new tokens
    pos = torch.arange(pm, device="cuda")
    cached = pos[None] < prefix[:, None]
    entry = torch.where(cached, st["block_table"].long()[:, :max(1, -(-pm // page))].repeat_interleave(page, 1)[:, :pm], 0)
    k = torch.cat([st["k_pages"][entry, :, pos % page].float(), st["k_new"][at].float()], 1).transpose(1, 2)      # [rows, hkv, pm + t, d]
    v = torch.cat([st["v_pages"][entry, :, pos % page].float(), st["v_new"][at].float()], 1).transpose(1, 2)
    if st["parent"] is None:
        level = i[None].expand(rows, t)
        sees = (i[None, None] <= i[None, :, None]).expand(rows, t, t)
    else:
        parent = torch.where(there, st["parent"].long()[at], -1)
        step = (parent[..., None] == i[None, None]).float() + torch.eye(t, device="cuda")
        reach = _squared(_squared(_squared(_squared(_squared(_squared(step))))))
        sees, level = reach > 0, (reach.sum(-1) - 1).long()
    qpos, kpos = prefix[:, None] + level, torch.cat([pos[None].expand(rows, pm), prefix[:, None] + level], 1)
    mask = torch.cat([cached[:, None].expand(rows, t, pm), sees & there[:, None]], 2)
    if c["window"]:
        mask = mask & ((qpos[:, :, None] - kpos[:, None] < c["window"]) | (kpos[:, None] < c["sinks"]))
    q = st["q"][at].float().view(rows, t, hkv, heads // hkv, d).permute(0, 2, 3, 1, 4).reshape(rows, hkv, -1, d)
    score = (q @ k.transpose(2, 3)).view(rows, hkv, heads // hkv, t, pm + t) * (1.0 / math.sqrt(d))
    score = score.masked_fill(~mask[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    weight = torch.exp(score - top)
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(rows, hkv, -1, pm + t) @ v).view(rows, hkv, heads // hkv, t, d) / total
    lse = (top + torch.log(total))[..., 0]
    pick = there.reshape(-1).nonzero()[:, 0]
    out = out.permute(0, 3, 1, 2, 4).reshape(rows * t, heads, d)[pick].to(st["q"].dtype)
    return {"out": out, "lse": lse.permute(0, 3, 1, 2).reshape(rows * t, heads)[pick]}


def _plain_append(st):
    slot, page = st["slot_map"].long(), st["case"]["page"]
    st["k_pages"][:, slot // page, :, slot % page] = st["k_new"].transpose(0, 1)
    st["v_pages"][:, slot // page, :, slot % page] = st["v_new"].transpose(0, 1)
    return {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_slots(st):
    length, page, table = st["seq_len"].long(), st["case"]["page"], st["block_table"]
    rows, width = table.shape
    new = st["new_len"].long() if st["new_len"] is not None else 1 + st["accept_len"].long()[st["row_prompt"].long()]
    have, end = (length + page - 1) // page, (length + new + page - 1) // page
    need = end - have
    before = torch.cumsum(need, 0) - need
    off = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)])
    e = torch.arange(width, device="cuda")
    taken = st["free_count"].long() - 1 - (before[:, None] + e[None] - have[:, None])
    fresh = (e[None] >= have[:, None]) & (e[None] < end[:, None])
    table = torch.where(fresh, st["free_pages"][torch.where(fresh, taken, 0)], table)
    t = torch.arange(st["slot_map"].numel(), device="cuda")
    row = torch.searchsorted(off[1:].contiguous(), t, right=True)
    used = row < rows
    row = torch.where(used, row, 0)
    j = t - off[row]
    pos = length[row] + j
    slot = table.long()[row, torch.where(used, pos // page, 0)] * page + pos % page
    if st["new_len"] is None:
        path = torch.cat([torch.zeros_like(st["path_nodes"][:, :1]), st["path_nodes"]], 1).long()
        source = st["node_off"].long()[row] + path[st["row_prompt"].long()[row], torch.where(used, j, 0)]
    else:
        source = t
    whole = lambda x: torch.where(used, x, -1).int()  # noqa: E731
    return {"q_off": off.int(), "slot_map": whole(slot), "position": whole(pos), "source": whole(source), "seq_len_out": (length + new).int(),
            "free_count_out": (st["free_count"].long() - need.sum()).int(), "block_table": table}


def _plain_sample(st):
    x = st["logits"].double()
    rows, vocab = x.shape
    greedy = ~(st["temperature"] > 0)
    t = torch.where(greedy, 1.0, st["temperature"].double())
    k = torch.where(st["top_k"] > 0, st["top_k"].long().clamp(max=vocab), vocab)
    k = torch.where(greedy, 1, k)
    ordered = torch.sort(x, dim=1, descending=True).values
    top = ordered[:, :1]
    least = ordered.gather(1, k[:, None] - 1)                                   # the k-th largest
    mass = torch.where(ordered >= least, torch.exp((ordered - top) / t[:, None]), 0.0)
    running = torch.cumsum(mass, 1)
    # the first place where the running mass reaches its share
    place = (running < st["top_p"].double()[:, None] * running[:, -1:]).sum(1, keepdim=True).clamp(max=vocab - 1)
    least = torch.where((st["top_p"] < 1)[:, None], torch.maximum(least, ordered.gather(1, place)), least)
    w = torch.exp((x - top) / t[:, None])
    w = torch.where((x >= least) & (w >= st["min_p"].double()[:, None]), w, 0.0)
    running = torch.cumsum(w, 1)
    token = (running <= st["u"].double()[:, None] * running[:, -1:]).sum(1).clamp(max=vocab - 1)
    lowest = torch.where(x == top, torch.arange(vocab, device="cuda")[None], vocab).amin(1)
    token = torch.where(greedy, lowest, token)
    prob = torch.where(greedy, 1.0, w.gather(1, token[:, None])[:, 0] / running[:, -1])
    return {"token": token.int(), "prob": prob.float()}


_RUN_OWN = {"attn": _own_attn, "append": _own_append, "slots": _own_slots, "sample": _own_sample}
_RUN_PLAIN = {"attn": _plain_attn, "append": _plain_append, "slots": _plain_slots, "sample": _plain_sample}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * size + 28), "flops": 2 * case["rows"] * case["vocab"]}
    prefix, new = _lengths(case)
    if case["kind"] == "slots":
        page, n = case["page"], sum(new)
        entries = sum(-(-(p + t) // page) - p // page for p, t in zip(prefix, new))
        places = case["rows"] * (case["depth"] + 1) if case["path"] else n
        return {"bytes": 4 * (4 * case["rows"] + 2 * entries + 3 * places), "flops": 4 * n}
    if case["kind"] == "append":
        return {"bytes": 4 * case["layers"] * sum(new) * case["kv_heads"] * case["head_dim"] * size + 4 * sum(new), "flops": 0}
    w, sinks, hkv, d = case["window"], case["sinks"], case["kv_heads"], case["head_dim"]
    keys = pairs = 0
    rng = random.Random(case["shape_seed"] + 1)
    for p, t in zip(prefix, new):
        if case["tree"]:
            level = [0]
            for a in _tree(rng, t, case["depth"])[1:]:
                level.append(level[a] + 1)
        else:
            level = range(t)
        for x in level:
            all_keys = p + x + 1
            pairs += min(all_keys, w + min(sinks, max(0, all_keys - w))) if w else all_keys
        keys += t + (min(p, max(0, w - 1) + min(sinks, max(0, p - w + 1))) if w else p)
    n = sum(new)
    return {"bytes": 2 * keys * hkv * d * size + 2 * n * case["heads"] * d * size + 4 * n * case["heads"] + 4 * keys // case["page"],
            "flops": 4 * d * case["heads"] * pairs}


def exact(case, seed):
    """The definitions in 64 bits, row by row."""
    if case["kind"] not in ("attn", "sample"):
        return None                                     # copies and whole numbers
    st = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(st)
    off, prefix, page = st["q_off"].tolist(), st["prefix_len"].tolist(), case["page"]
    table = st["block_table"].cpu().numpy()
    parent = None if st["parent"] is None else st["parent"].cpu().numpy()
    group = case["heads"] // case["kv_heads"]
    out, lse = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for s in range(case["rows"]):
        lo, hi, p = off[s], off[s + 1], prefix[s]
        where = np.arange(p)
        pg = torch.from_numpy(table[s, where // page].astype(np.int64)).cuda()
        inside = torch.from_numpy(where % page).cuda()
        sees, level = np.zeros((hi - lo, hi - lo), bool), np.zeros(hi - lo, np.int64)
        for i in range(hi - lo):
            if parent is None:
                sees[i, :i + 1], level[i] = True, i
            else:
                a = int(parent[lo + i])
                if a >= 0:
                    sees[i], level[i] = sees[a], level[a] + 1
                sees[i, i] = True
        qp, kp = p + level, np.concatenate([where, p + level])
        seen = np.concatenate([np.ones((hi - lo, p), bool), sees], 1)
        if case["window"]:
            seen &= (qp[:, None] - kp[None] < case["window"]) | (kp[None] < case["sinks"])
        seen = torch.from_numpy(seen).cuda()
        for h in range(case["kv_heads"]):
            key = torch.cat([st["k_pages"][pg, h, inside], st["k_new"][lo:hi, h]]).double()
            val = torch.cat([st["v_pages"][pg, h, inside], st["v_new"][lo:hi, h]]).double()
            for x in range(h * group, (h + 1) * group):
                z = (st["q"][lo:hi, x].double() @ key.T / math.sqrt(case["head_dim"])).masked_fill(~seen, -math.inf)
                lse[lo:hi, x] = torch.logsumexp(z, 1)
                out[lo:hi, x] = torch.softmax(z, 1) @ val
    return {"out": out, "lse": lse}


def _exact_sample(st):
    rows = st["logits"].double().cpu().numpy()
    par = {k: st[k].double().cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p", "u")}
    token, prob = [], []
    for r, x in enumerate(rows):
        t, k, p, least, u = (float(par[key][r]) for key in ("temperature", "top_k", "top_p", "min_p", "u"))
        if not t > 0:
            token.append(int(np.flatnonzero(x == x.max())[0]))
            prob.append(1.0)
            continue
        w = np.exp((x - x.max()) / t)
        keep = np.ones(len(x), bool)
        if 0 < k < len(x):
            keep = x >= np.partition(x, len(x) - int(k))[len(x) - int(k)]
        if p < 1:
            values, which = np.unique(x[keep], return_inverse=True)
            above = np.cumsum(np.bincount(which, weights=w[keep])[::-1])        # mass of what is at least so large, largest value first
            keep &= x >= values[::-1][min(int(np.searchsorted(above, p * w[keep].sum())), len(values) - 1)]
        keep &= w >= least
        w = np.where(keep, w, 0.0)
        run_ = np.cumsum(w)
        at = int(np.searchsorted(run_, u * run_[-1], side="right"))
        token.append(at)
        prob.append(w[at] / run_[-1])
    return {"token": np.array(token, np.int32), "prob": np.array(prob)}
