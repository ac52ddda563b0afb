"""Problems for the calls on pages that rows share and on caches that are held to a budget, and their comparison with the oracle."""
import numpy as np
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding

from serving_util import DT, ORDERS, Problem, dev


class Shared(Problem):
    """Rows of a group hold the pages of its first row for the first `shared` positions; the pages that they would have had for them are NaN."""

    def __init__(self, seed, prefix, new, groups, shared, **kw):
        super().__init__(seed, prefix, new, **kw)
        self.groups, self.shared = groups, shared
        for g, (lo, hi) in enumerate(zip(groups, groups[1:])):
            n = max(shared[g], 0) // self.page
            for s in range(lo + 1, hi):
                m = min(n, -(-prefix[s] // self.page), prefix[lo] // self.page)          # (a shorter row: all of its pages)
                dropped = self.table[s, :m]
                dropped = dropped[dropped < self.k_pages.shape[0]]          # (a window has passed the others: they name no page)
                assert ((dropped >= 0) & (dropped < self.k_pages.shape[0])).all()
                for pages in (self.k_pages, self.v_pages):
                    pages[dev(dropped, np.int64)] = float("nan")
                self.table[s, :m] = self.table[lo, :m]
        self.args["block_table"] = self.block_table = dev(self.table)
        self.args.update(group_off=dev(groups), shared_len=dev(shared), max_shared_len=max(0, min(max(shared), max(prefix))))

    def run(self, ctx=None, **more):
        binding.paged_attn_shared(ctx or self.context(), **{**self.args, "out": self.out, "lse": self.lse, **more})
        torch.cuda.synchronize()

    def cut(self, ctx=None):
        return binding.paged_shared_cut(n_rows=len(self.prefix), n_groups=len(self.shared), n_tokens=self.n, max_new=self.args["max_new"],
                                        max_prefix_len=self.args["max_prefix_len"], max_shared_len=self.args["max_shared_len"], n_heads=self.heads,
                                        n_kv_heads=self.kv_heads, head_dim=self.head_dim, tree=self.parent is not None, window=self.window,
                                        dtype=binding.BF16 if self.dtype == "bf16" else binding.F32, ctx=ctx)


class Mass:
    """New tokens at the end of some rows, all keys in pages.  Places of the pool that hold no position are NaN, entries of the table that no token needs
    are far outside the pool."""

    def __init__(self, seed, length, new, *, heads=8, kv_heads=4, head_dim=128, dtype="bf16", page=16, order="head", window=0, n_sink=0, first=None, path=0,
                 spare=0, packed=False, scale=0.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        randn = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(DT[dtype])  # noqa: E731
        self.length, self.new, self.page, self.window, self.n_sink, self.dtype = length, new, page, window, n_sink, dtype
        self.heads, self.kv_heads, self.head_dim, self.scale = heads, kv_heads, head_dim, scale
        rows, n = len(length), sum(new)
        self.off = np.concatenate([[0], np.cumsum(new)])
        self.first = first if first is not None else [0] * rows
        drafted = n + path + spare
        self.q = randn(drafted, heads + (2 * kv_heads if packed else 0), head_dim)[:, :heads]
        self.lse = (torch.rand(drafted, heads, device="cuda", generator=gen) * 3 + 2).contiguous()
        self.source = np.sort(rng.permutation(drafted)[:n]) if path else np.arange(n)
        held = [-(-x // page) for x in length]
        pool = sum(held) + 3
        ids = rng.permutation(pool)
        table = np.full((rows, max(max(held), 1) + 2), 1 << 30, np.int64)
        used = torch.zeros(pool, page, dtype=torch.bool)
        at = 0
        for s, x in enumerate(length):
            before = x - new[s]
            for e in range(held[s]):
                g = ids[at]
                at += 1
                reach = max(0, before - window + 1) if window else 0
                if new[s] == 0 or ((e + 1) * page <= reach and e * page >= n_sink) or (e + 1) * page <= self.first[s]:
                    continue
                table[s, e] = g
                used[g, :min(page, x - e * page)] = True
        perm = ORDERS[order]
        shape = (pool, kv_heads, page, head_dim)
        self.k_pages = randn(*(shape[i] for i in perm)).permute(*np.argsort(perm))
        self.k_pages.masked_fill_(~used.cuda()[:, None, :, None], float("nan"))
        self.table = table
        self.mass = torch.rand(rows, kv_heads, max(length) + 7, device="cuda", generator=gen)
        for s in range(rows):                                    # what stands where the new tokens' sums go is not read
            self.mass[s, :, length[s] - new[s]:length[s]] = float("nan")
        self.before = self.mass.clone()
        self.args = dict(q_off=dev(self.off), seq_len=dev(length), block_table=dev(table)[:, :max(max(held), 1)], q=self.q, lse=self.lse, k_pages=self.k_pages,
                         mass=self.mass, source=dev(self.source) if path else None, first=dev(first) if first is not None else None, window=window, n_sink=n_sink,
                         max_new=max(new), max_seq_len=max(length), scale=scale)

    def context(self, stream=None):
        return binding.Context(max_rows=len(self.length), max_nodes_total=max(1, self.q.shape[0]), max_nodes_per_tree=1, max_prefix=max(self.length), n_heads=self.heads,
                               head_dim=self.head_dim, hidden=64, vocab=64, stream=stream)

    def run(self, ctx=None, **more):
        binding.paged_mass(ctx or self.context(), **{**self.args, **more})
        torch.cuda.synchronize()

    def check(self, rows=None):
        """A score's error d (float32 products of head_dim terms; the difference to lse, in units of log 2, rounded twice) moves its exponential by d, relative;
        the exponential itself and the sums add (terms + 64) 2^-24."""
        group = self.heads // self.kv_heads
        got, old = self.mass.double().cpu().numpy(), self.before.double().cpu().numpy()
        for s in range(len(self.length)) if rows is None else rows:
            length, n, first = self.length[s], self.new[s], min(max(self.first[s], 0), self.length[s])
            before = length - n
            assert np.array_equal(got[s, :, length:], old[s, :, length:]), (s, "behind the row")
            assert np.array_equal(got[s, :, :first], old[s, :, :first], equal_nan=True), (s, "in front of first")
            if n == 0:
                assert np.array_equal(got[s], old[s], equal_nan=True)
                continue
            tokens = self.source[self.off[s]:self.off[s + 1]]
            pos = np.arange(length)
            x = before + np.arange(n)
            sees = pos[None] <= x[:, None]
            if self.window:
                sees &= (x[:, None] - pos[None] < self.window) | (pos[None] < self.n_sink)
            entry = self.table[s, pos // self.page]
            bad = (entry < 0) | (entry >= self.k_pages.shape[0])
            for h in range(self.kv_heads):
                k = self.k_pages[dev(np.where(bad, 0, entry), np.int64), h, dev(pos % self.page, np.int64)].double().cpu().numpy()
                k[bad] = np.nan
                ok = sees & ~bad[None]
                at = dev(tokens, np.int64)
                q, lse = (t[at, h * group:(h + 1) * group].double().cpu().numpy() for t in (self.q, self.lse))
                want, size = so.attention_mass(q, lse, k, ok, self.scale or None)
                tol = want * ((n * group + 64) * 2.0 ** -24) + size * (self.head_dim + 20) * 2.0 ** -24 + 1e-37
                total = np.where(pos < before, np.where(bad, old[s, h, :length], old[s, h, :length] + want), want)
                tol += 2.0 ** -24 * np.abs(total)
                a, b, t = got[s, h, first:length], total[first:], tol[first:]
                fine = np.isfinite(b)
                assert np.array_equal(np.isfinite(a), fine), (s, h, "finite places differ", np.argwhere(np.isfinite(a) != fine)[:4])
                assert (np.abs(a - b)[fine] <= t[fine]).all(), (s, h, float((np.abs(a - b)[fine] / t[fine]).max()))


class Evict:
    """Rows of several lengths, every layer and head with weights of its own, many of them equal.  Keys are numbers of their places."""

    def __init__(self, seed, length, budget, *, layers=2, kv_heads=3, head_dim=64, dtype="bf16", page=16, first=None, recent=0, free=3, order=(0, 1, 2, 3, 4), levels=40,
                 cap=None):
        rng = np.random.default_rng(seed)
        self.length, self.budget, self.first, self.recent, self.page, self.dtype = length, budget, first, recent, page, dtype
        rows = len(length)
        held = [-(-max(x, 0) // page) for x in length]
        pool = sum(held) + free + 2
        ids = rng.permutation(pool)
        self.table = np.full((rows, max(max(held), 1)), 1 << 30, np.int64)
        at = 0
        for s in range(rows):
            self.table[s, :held[s]] = ids[at:at + held[s]]
            at += held[s]
        self.free = np.concatenate([ids[at:at + free], np.full(pool - free, -5)])
        self.n_free = free
        shape = (layers, pool, kv_heads, page, head_dim)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        make = lambda: torch.randn([shape[i] for i in order], device="cuda", generator=gen).to(DT[dtype]).permute(*np.argsort(order))  # noqa: E731
        self.k_pages, self.v_pages = make(), make()
        cap = cap or max(max(length), 1) + 3
        mass = rng.integers(0, levels, (layers, rows, kv_heads, cap)).astype(np.float32) / 8
        self.mass = torch.from_numpy(mass).cuda()
        self.mass_out = torch.full_like(self.mass, -7.0)
        one = lambda n: torch.full((n,), -9, dtype=torch.int32, device="cuda")  # noqa: E731
        self.args = dict(seq_len=dev(length), budget=dev(budget), block_table=dev(self.table), k_pages=self.k_pages, v_pages=self.v_pages, mass=self.mass, mass_out=self.mass_out,
                         free_pages=dev(self.free), free_count=dev([free]), seq_len_out=one(rows), free_count_out=one(1), dropped=one(rows),
                         n_first=None if first is None else dev(first), n_recent=recent, max_seq_len=max(max(length), 0))
        self.was = [t.clone() for t in (self.k_pages, self.v_pages, self.mass)]

    def context(self, stream=None):
        return binding.Context(max_rows=len(self.length), max_nodes_total=1, max_nodes_per_tree=1, max_prefix=max(1, self.args["max_seq_len"]), n_heads=8,
                               head_dim=self.k_pages.shape[4], hidden=64, vocab=64, stream=stream)

    def workspace(self, ctx, **more):
        size = binding.paged_evict_workspace(ctx, **{**self.args, **{k: v for k, v in more.items() if k != "workspace"}})
        return torch.empty(size, dtype=torch.uint8, device="cuda") if size else None

    def run(self, ctx=None, **more):
        ctx = ctx or self.context()
        if "workspace" not in more:
            more["workspace"] = self.workspace(ctx, **more)
        binding.paged_evict(ctx, **{**self.args, **more})
        torch.cuda.synchronize()

    def check(self, skip=()):
        """Every place of the pool, of the weights, of the lists: those that the definition does not name are as they were."""
        k, v, mass = (t.cpu().numpy() if t.dtype == torch.float32 else t.view(torch.int16).cpu().numpy() for t in self.was)
        want_k, want_v = k.copy(), v.copy()
        want_mass = np.full(mass.shape, -7.0, np.float32)
        back, lengths = [], []
        for s, n in enumerate(self.length):
            if s in skip:
                lengths.append(n)
                continue
            f = self.first[s] if self.first is not None else 0
            for layer in range(mass.shape[0]):
                for h in range(mass.shape[2]):
                    place = np.array(so.evict_places(mass[layer, s, h], n, self.budget[s], f, self.recent), np.int64)
                    after = len(place)
                    want_mass[layer, s, h, :after] = mass[layer, s, h, place]
                    to = np.flatnonzero(place != np.arange(after))
                    src, dst = place[to], to
                    a = (layer, self.table[s, dst // self.page], h, dst % self.page)
                    b = (layer, self.table[s, src // self.page], h, src % self.page)
                    want_k[a], want_v[a] = k[b], v[b]
            lengths.append(after)
            back += self.table[s, -(-after // self.page):-(-n // self.page)].tolist()
        for name, want, got in (("k", want_k, self.k_pages), ("v", want_v, self.v_pages)):
            got = got.cpu().numpy() if got.dtype == torch.float32 else got.view(torch.int16).cpu().numpy()
            assert np.array_equal(got, want), (name, np.argwhere(got != want)[:3])
        assert np.array_equal(self.mass_out.cpu().numpy(), want_mass, equal_nan=True)
        assert np.array_equal(self.mass.cpu().numpy(), mass, equal_nan=True)
        a = self.args
        assert a["seq_len_out"].tolist() == lengths
        assert a["dropped"].tolist() == [0 if s in skip else n - m for s, (n, m) in enumerate(zip(self.length, lengths))]
        assert a["free_count_out"].tolist() == [self.n_free + len(back)]
        want_free = self.free.copy()
        want_free[self.n_free:self.n_free + len(back)] = back
        assert a["free_pages"].tolist() == want_free.tolist()
