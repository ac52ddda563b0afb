"""PagedLoop with rows that begin in the same pages and are held to a budget: prompts, shared pages, steps, evictions and further steps chained, against a mirror of every
row's keys and values per kv head, kept on the host."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding
from paper_2605_07230_amd import decode
from paper_2605_07230_amd import workloads as wl

pytestmark = pytest.mark.gpu
PAGE = 16


def _inputs(dtype, prompts, heads, kv_heads, nodes, head_dim=64):
    rng = np.random.default_rng(5)
    return wl.make_inputs(name="paged_loop_budget", seed=12, dtype=dtype, n_prompts=prompts, cfg=False, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, hidden=256,
                          vocab=4096, prefix_lens=[8] * prompts, trees=[wl.grow_tree(rng, nodes, 4, 8) for _ in range(prompts)], cfg_scale=1.0, temperature=1.0,
                          top_k=200, tau_pos=0.8, tau_seq=0.5, eps_tvd=0.5, token_law="zipf")


class Mirror:
    """What each row holds, a list of positions for each kv head, as bits."""

    def __init__(self, loop):
        self.loop = loop
        self.keys = [[[] for _ in range(loop.inp.n_kv_heads)] for _ in range(loop.rows)]

    def add(self, s, k, v):                       # k, v: [tokens, kv heads, d]
        for h, held in enumerate(self.keys[s]):
            held += [(k[t, h], v[t, h]) for t in range(len(k))]

    def check(self):
        loop = self.loop
        lens = loop.seq_len.tolist()
        for s, row in enumerate(self.keys):
            assert lens[s] == len(row[0]), s
            pages = loop.block_table[s, :-(-lens[s] // PAGE)].long()
            for i, pool in enumerate((loop.k_pages, loop.v_pages)):
                got = pool[0, pages].transpose(1, 2).reshape(-1, *pool.shape[2:3], pool.shape[4])[:lens[s]].double().cpu().numpy()
                for h, held in enumerate(row):
                    if held:
                        assert np.array_equal(got[:, h], np.stack([x[i] for x in held])), (s, h, "kv"[i])

    def attention(self, s, h, q, k_new, v_new, parent):
        k = np.stack([x[0] for x in self.keys[s][h]] + list(k_new))
        v = np.stack([x[1] for x in self.keys[s][h]] + list(v_new))
        return so.attention(q, k, v, so.visible(len(self.keys[s][h]), len(q), parent))


@pytest.mark.parametrize("dtype,shares", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_the_chain(dtype, shares):
    # enough rows and shared keys that the shared pass runs, or few
    prompts, heads, kv_heads, n_shared, nodes, dim = (34, 32, 16, 960, 6, 128) if shares and dtype == "bf16" else (24, 2, 2, 512, 5, 64) if shares else (5, 4, 2, 64, 20, 64)
    inp = _inputs(dtype, prompts, heads, kv_heads, nodes, dim)
    print(f"[paged loop budget] {dtype} shared pass {shares}", flush=True)
    loop = decode.PagedLoop(inp, page_size=PAGE, max_len=n_shared + 160, max_chunk=n_shared + 30, n_pages=prompts * 12 + 2 * n_shared // PAGE + 8, keep_mass=True)
    S, st, mirror = loop.rows, loop.step_in, Mirror(loop)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    mk = lambda n, h: torch.randn(n, h, inp.head_dim, device="cuda", generator=gen).to(st.q.dtype)  # noqa: E731
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    some = sorted({0, 1, S // 2, S - 1})
    heads_seen = (0, heads - 1)

    def fine(out, ref, mag, size, n):
        tol = mag * (2 * half + 2 * (inp.head_dim + 16) * 2.0 ** -24 * (1 + size[:, None]) + (n + 64) * 2.0 ** -23) + half * np.abs(ref) + 1e-30
        assert (np.abs(out - ref) <= tol).all(), float((np.abs(out - ref) / tol).max())

    def admit(new):
        n = sum(new)
        q, k, v = mk(n, heads), mk(n, kv_heads), mk(n, kv_heads)
        out = torch.empty_like(q)
        loop.admit(q, k, v, new, out)
        torch.cuda.synchronize()
        off = np.concatenate([[0], np.cumsum(new)])
        for s in range(S):
            a, b = off[s], off[s + 1]
            if s in some and b > a:
                for x in heads_seen:
                    h = x * kv_heads // heads
                    ref, _, mag, size = mirror.attention(s, h, host(q[a:b, x]), host(k[a:b, h]), host(v[a:b, h]), None)
                    fine(host(out[a:b, x]), ref, mag, size, b - a + n_shared)
            mirror.add(s, host(k[a:b]), host(v[a:b]))

    # two groups whose prompts are the first rows' to begin with; the last row is by itself
    groups, given = [0, S // 2, S - 1, S], [n_shared, n_shared - PAGE, 0]
    admit([n_shared + 5 if s == 0 else n_shared - PAGE if s == S // 2 else 0 for s in range(S)])
    loop.share(groups, given)
    for lo, hi, n in zip(groups, groups[1:], given):
        for s in range(lo + 1, hi):
            for h in range(kv_heads):
                mirror.keys[s][h] = list(mirror.keys[lo][h][:n])
    mirror.check()
    admit([10 + s % 7 for s in range(S)])
    mirror.check()
    first = [given[0] if s < S // 2 else given[1] if s < S - 1 else 0 for s in range(S)]
    assert loop.held.tolist() == first
    if shares:
        assert binding.paged_shared_cut(n_rows=S, n_groups=3, n_tokens=st.q.shape[0], max_new=st.max_tree, max_prefix_len=loop.longest, max_shared_len=n_shared, n_heads=heads,
                                        n_kv_heads=kv_heads, head_dim=inp.head_dim, tree=True, dtype=binding.BF16 if dtype == "bf16" else binding.F32, ctx=loop.ctx)[1] > 0

    def steps(count):
        for _ in range(count):
            before = [[list(x) for x in row] for row in mirror.keys]
            mass = host(loop.mass[0])
            loop.step()
            torch.cuda.synchronize()
            node, parent = st.row_node_off.tolist(), st.row_parent.cpu().numpy()
            q, k, v, out, lse = (host(t) for t in (st.q, st.k_tree, st.v_tree, st.attn_out, st.attn_lse))
            got = host(loop.mass[0])
            for s in range(S):
                a, b = node[s], node[s + 1]
                for x in heads_seen if s in some else ():
                    h = x * kv_heads // heads
                    ref, _, mag, size = mirror.attention(s, h, q[a:b, x], k[a:b, h], v[a:b, h], parent[a:b])
                    fine(out[a:b, x], ref, mag, size, len(before[s][h]) + nodes)
                path = [0] + [p for p in st.path_nodes[s].tolist() if p >= 0][:int(st.accept_len[s])]
                mirror.add(s, k[a:b][path], v[a:b][path])
                if s in some:                     # the gathered weights: behind what is held, of the kept path alone
                    for h in (0, kv_heads - 1):
                        g = heads // kv_heads
                        keys = np.stack([x[0] for x in mirror.keys[s][h]])
                        n, new = len(keys), len(path)
                        sees = np.arange(n)[None] <= (n - new + np.arange(new))[:, None]
                        want, size = so.attention_mass(q[a:b][path][:, h * g:(h + 1) * g], lse[a:b][path][:, h * g:(h + 1) * g], keys, sees)
                        total = want + np.where(np.arange(n) < n - new, mass[s, h, :n], 0)
                        tol = (want * (n + 64) + size * (inp.head_dim + 20) + total) * 2.0 ** -24 + 1e-30
                        assert (np.abs(got[s, h, first[s]:n] - total[first[s]:]) <= tol[first[s]:]).all(), (s, h)
                        assert np.array_equal(got[s, h, :first[s]], mass[s, h, :first[s]])
            mirror.check()

    def evict(budget, n_first, n_recent):
        mass, free = host(loop.mass[0]), int(loop.free_count)
        held = [len(mirror.keys[s][0]) for s in range(S)]
        loop.evict(budget, n_first=n_first, n_recent=n_recent)
        torch.cuda.synchronize()
        now = host(loop.mass[0])
        back = 0
        for s in range(S):
            for h in range(kv_heads):
                place = so.evict_places(mass[s, h], held[s], budget if isinstance(budget, int) else budget[s], max(first[s], n_first), n_recent)
                mirror.keys[s][h] = [mirror.keys[s][h][y] for y in place]
                assert np.array_equal(now[s, h, :len(place)], mass[s, h, place])
            back += -(-held[s] // PAGE) - -(-len(place) // PAGE)
        assert int(loop.free_count) == free + back
        mirror.check()
        return sum(held) - sum(len(row[0]) for row in mirror.keys)

    steps(2)
    gone = evict([f + 12 for f in first], 0, 5)
    assert gone > S and int(loop.dropped.sum()) == gone
    steps(2)
    gone += evict(n_shared + 10, 3, 8)
    steps(1)
    assert int(loop.dropped.sum()) == gone
    # pages: those that rows share once, the others each their own
    ends = loop.seq_len.tolist()
    used = [p for s in range(S) for p in loop.block_table[s, (first[s] // PAGE if s not in groups else 0):-(-ends[s] // PAGE)].tolist()]
    assert len(set(used)) == len(used) == loop.n_pages - int(loop.free_count)
    assert loop.ctx.device_status() == binding.OK


def test_rows_without_pages_are_not_weighed():
    inp = _inputs("bf16", 3, 4, 2, 5)
    loop = decode.PagedLoop(inp, page_size=PAGE, max_len=320, max_chunk=100, n_pages=9, keep_mass=True)
    mk = lambda n, h: torch.randn(n, h, inp.head_dim, device="cuda").bfloat16()  # noqa: E731
    for new, ends in (([40, 30, 20], [40, 30, 20]), ([17, 60, 1], [57, 30, 21])):
        n = sum(new)
        q = mk(n, 4)
        before = loop.mass.clone()
        loop.admit(q, mk(n, 2), mk(n, 2), new, torch.empty_like(q))
        torch.cuda.synchronize()
        assert loop.seq_len.tolist() == ends
    assert loop.ctx.device_status() == binding.ETREE            # no pages for the second row's second chunk
    assert torch.equal(loop.mass[0, 1], before[0, 1])
    for s, count in ((0, 57), (2, 21)):                         # every token's weights sum to one for each of its query heads
        assert torch.allclose(loop.mass[0, s].sum(1), torch.full((2,), 2.0 * count, device="cuda"), rtol=1e-4)


def test_refusals():
    inp = _inputs("bf16", 4, 4, 2, 5)
    loop = decode.PagedLoop(inp, page_size=PAGE, max_len=320, max_chunk=100, keep_mass=True)
    plain = decode.PagedLoop(inp, page_size=PAGE, max_len=320, max_chunk=100)
    with pytest.raises(ValueError):
        plain.evict(10)
    q = torch.randn(70, 4, inp.head_dim, device="cuda").bfloat16()
    kv = torch.randn(70, 2, inp.head_dim, device="cuda").bfloat16()
    loop.admit(q, kv, kv, [64, 0, 6, 0], torch.empty_like(q))
    for groups, n in (([0, 2, 4], [64]), ([0, 2, 3], [64, 0]), ([1, 2, 4], [64, 0]), ([0, 3, 2, 4], [0, 0, 0]), ([0, 2, 4], [60, 0]), ([0, 2, 4], [80, 0]), ([0, 2, 4], [-16, 0]),
                      ([0, 4], [64])):
        with pytest.raises(ValueError):
            loop.share(groups, n)
    loop.share([0, 2, 4], [48, 0])
    with pytest.raises(ValueError):
        loop.share([0, 2, 4], [48, 0])
    for args in (([5, 5, 5],), (-1,), (5, -1), (5, 0, -1)):
        with pytest.raises(ValueError):
            loop.evict(*args)
    torch.cuda.synchronize()
    assert loop.seq_len.tolist() == [64, 48, 6, 0] and loop.ctx.device_status() == binding.OK
    again = decode.PagedLoop(inp, page_size=PAGE, max_len=320, max_chunk=100, keep_mass=True)
    again.admit(q, kv, kv, [64, 0, 6, 0], torch.empty_like(q))
    again.evict(50)
    with pytest.raises(ValueError):                             # heads of the first row hold positions of their own by now
        again.share([0, 2, 4], [48, 0])
