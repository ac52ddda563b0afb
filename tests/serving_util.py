"""Random problems for the calls on pages, and their comparison with the oracle."""
import numpy as np
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding
from paper_2605_07230_amd import workloads as wl

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ORDERS = {"head": (0, 1, 2, 3), "position": (0, 2, 1, 3), "page_inside": (1, 0, 2, 3)}    # memory order of (page, head, position, d)


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


class Problem:
    """New tokens of some rows over a cache in pages.  Places of the pool that hold no position are NaN, entries of the table behind a row's pages
    (and, with a window, in front of it) are far outside the pool."""

    def __init__(self, seed, prefix, new, *, heads=8, kv_heads=8, head_dim=128, dtype="bf16", page=16, order="head", tree=False, window=0, n_sink=0,
                 spare=0, packed_qkv=False, scale=0.0, q_scale=1.0):
        rng = np.random.default_rng(seed)
        self.prefix, self.new, self.page, self.window, self.n_sink, self.scale, self.dtype = prefix, new, page, window, n_sink, scale, dtype
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        randn = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(DT[dtype])  # noqa: E731
        self.n = n = sum(new) + spare                       # spare: tokens behind the last row
        self.off = np.concatenate([[0], np.cumsum(new)])
        if packed_qkv:                                      # one projection's output, sliced
            qkv = randn(n, heads + 2 * kv_heads, head_dim)
            self.q, self.k_new, self.v_new = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        else:
            self.q, self.k_new, self.v_new = randn(n, heads, head_dim), randn(n, kv_heads, head_dim), randn(n, kv_heads, head_dim)
        if q_scale != 1.0:
            self.q = self.q * q_scale
        held = [-(-p // page) for p in prefix]
        pool = sum(held) + 3
        ids = rng.permutation(pool)
        width = max(max(held), 1)
        table = np.full((len(prefix), width + 2), 1 << 30, np.int64)
        used = torch.zeros(pool, page, dtype=torch.bool)
        at = 0
        for s, p in enumerate(prefix):
            for e in range(held[s]):
                g = ids[at]
                at += 1
                first = max(0, p - window + 1) if window else 0        # the first position that a token of the row sees, sinks apart
                if (e + 1) * page <= first and e * page >= min(n_sink, p):
                    continue
                table[s, e] = g
                used[g, :min(page, p - e * page)] = True
        perm = ORDERS[order]
        shape = (pool, kv_heads, page, head_dim)
        pools = []
        for _ in range(2):
            t = randn(*(shape[i] for i in perm)).permute(*np.argsort(perm))
            t.masked_fill_(~used.cuda()[:, None, :, None], float("nan"))
            pools.append(t)
        self.k_pages, self.v_pages = pools
        self.table = table[:, :width]
        self.block_table = dev(table)[:, :width]
        self.parent = None
        if tree:
            self.parent = np.concatenate([wl.grow_tree(rng, t, min(tree, max(t - 1, 0)), 10) if t > 1 else np.array([-1]) for t in new]).astype(np.int32)
        self.args = dict(q_off=dev(self.off), prefix_len=dev(prefix), block_table=self.block_table, q=self.q, k_new=self.k_new, v_new=self.v_new,
                         k_pages=self.k_pages, v_pages=self.v_pages, parent=None if self.parent is None else dev(np.concatenate([self.parent, np.full(spare, -1)])),
                         window=window, n_sink=n_sink, max_new=max(new), max_prefix_len=max(prefix), scale=scale)
        self.out = torch.full((n, heads, head_dim), 7.0, device="cuda", dtype=DT[dtype])
        self.lse = torch.full((n, heads), 7.0, device="cuda")
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim

    def context(self, stream=None):
        return binding.Context(max_rows=len(self.prefix), max_nodes_total=self.n, max_nodes_per_tree=max(1, min(1024, max(self.new), self.n)),
                               max_prefix=max(self.prefix), n_heads=self.heads, head_dim=self.head_dim, hidden=64, vocab=64, stream=stream)

    def run(self, ctx=None, **more):
        binding.paged_attn(ctx or self.context(), **{**self.args, "out": self.out, "lse": self.lse, **more})
        torch.cuda.synchronize()

    def row_keys(self, s, h):
        """All keys and values of row s, kv head h, in order; a place that no token may see: as it lies, NaN."""
        p, lo, hi = self.prefix[s], self.off[s], self.off[s + 1]
        pos = np.arange(p)
        g = self.table[s, pos // self.page]
        bad = g >= self.k_pages.shape[0]
        at = dev(np.where(bad, 0, g), np.int64), dev(pos % self.page, np.int64)
        out = []
        for pages, fresh in ((self.k_pages, self.k_new), (self.v_pages, self.v_new)):
            x = pages[at[0], h, at[1]].double()
            x[dev(bad, bool)] = float("nan")
            out.append(torch.cat([x, fresh[lo:hi, h].double()]).cpu().numpy())
        return out

    def check(self, heads=None):
        """Every token of every row against the oracle.  A probability is rounded to the type (at most half a step, relative) where it enters
        the product, and a result when it is written.  A score's error d (float32
        products of head_dim terms) moves each probability by d.  What float32 sums add is counted as (keys + 64) 2^-24."""
        out, lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        half = 2.0 ** -8 if self.dtype == "bf16" else 0.0
        group = self.heads // self.kv_heads
        worst = 0.0
        for s in range(len(self.prefix)):
            lo, hi = self.off[s], self.off[s + 1]
            parent = None if self.parent is None else self.parent[lo:hi]
            sees = so.visible(self.prefix[s], hi - lo, parent, self.window, self.n_sink)
            for h in range(self.kv_heads) if heads is None else heads:
                k, v = self.row_keys(s, h)
                for g in range(h * group, (h + 1) * group):
                    ref, ref_lse, mag, size = so.attention(self.q[lo:hi, g].double().cpu().numpy(), k, v, sees, self.scale or None)
                    d = (self.head_dim + 16) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + np.abs(np.where(np.isfinite(ref_lse), ref_lse, 0)))
                    tol = mag * (half + 2 * d[:, None] + (len(k) + 64) * 2.0 ** -24) + half * np.abs(ref) + 1e-30
                    fine = np.isfinite(ref)
                    assert np.array_equal(np.isfinite(out[lo:hi, g]), fine), (s, g, "finite places differ")
                    err = np.abs(out[lo:hi, g] - ref)[fine] / tol[fine]
                    worst = max(worst, err.max(initial=0.0))
                    assert (err <= 1).all(), (s, g, float(err.max()), np.argwhere(np.abs(out[lo:hi, g] - ref) > tol)[:3])
                    ok = np.isfinite(ref_lse)
                    # sums are of probabilities that are not rounded to the type
                    assert (np.abs(lse[lo:hi, g] - ref_lse)[ok] <= (2 * d + (len(k) + 64) * 2.0 ** -24)[ok]).all(), (s, g, "lse")
        assert (self.out[self.off[-1]:] == 7).all() and (self.lse[self.off[-1]:] == 7).all()     # tokens behind the last row
        return worst
