"""paged_attn in every way the dispatcher cuts it (16 query rows with four or eight waves, 64 / 128 / 256 rows, keys whole or in parts, chains and trees, one or many items to a
workgroup, rows ranked or in order), at head_dim 64 and 128; every output of the heads looked at against float64, also with infinities and NaN among the values."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding

from serving_util import Problem, dev

pytestmark = pytest.mark.gpu


def _ragged(rows, most, least=0):
    """`rows` lengths between the two, none of them a round one by intent."""
    return [least + (most - least) * ((7 * s + 3) % 11) // 10 if s else most for s in range(rows)]


CASES = {
    "tokens, one part": dict(prefix=[312, 300], new=[1, 1], heads=8, kv_heads=8),
    "tokens, parts": dict(prefix=[3000, 700], new=[1, 2], heads=8, kv_heads=2),
    "tokens, full chip": dict(prefix=_ragged(300, 130), new=[1] * 300, heads=8, kv_heads=4),
    "tokens, full chip, parts": dict(prefix=_ragged(70, 1200, 40), new=_ragged(70, 3, 1), heads=16, kv_heads=8, page=32),
    "tokens, full chip, window": dict(prefix=_ragged(200, 300), new=_ragged(200, 2, 1), heads=12, kv_heads=4, window=70, n_sink=3),
    "small trees": dict(prefix=[600, 30], new=[7, 3], heads=4, kv_heads=2, tree=3),
    "small trees, parts": dict(prefix=[3000, 700], new=[8, 5], heads=4, kv_heads=2, tree=3),
    "small trees, full chip": dict(prefix=_ragged(180, 130), new=_ragged(180, 8, 1), heads=16, kv_heads=8, tree=3, window=90, n_sink=1),
    "64 rows": dict(prefix=[50, 77], new=[40, 33], heads=2, kv_heads=2),
    "64 rows, parts": dict(prefix=[1500, 37, 700], new=[60, 41, 17], heads=2, kv_heads=2, page=48),
    "64 rows, trees": dict(prefix=[50, 77], new=[40, 33], heads=2, kv_heads=2, tree=6),
    "64 rows, trees, parts": dict(prefix=[1500, 37, 700], new=[60, 41, 17], heads=2, kv_heads=2, tree=6),
    "many rows, in order": dict(prefix=_ragged(132, 90), new=_ragged(132, 10, 1), heads=32, kv_heads=4),
    "many rows, in order, trees": dict(prefix=_ragged(134, 90), new=_ragged(134, 10, 1), heads=32, kv_heads=4, tree=4),
    "chunks, ranked": dict(prefix=_ragged(16, 210), new=_ragged(16, 251, 7), heads=16, kv_heads=4),
    "chunks, ranked, window": dict(prefix=_ragged(16, 410), new=_ragged(16, 251, 7), heads=16, kv_heads=4, window=90, n_sink=5, page=32),
    "chunks, ranked, trees": dict(prefix=_ragged(16, 210), new=_ragged(16, 251, 7), heads=16, kv_heads=4, tree=12),
    "chunks, ranked, trees, window": dict(prefix=_ragged(16, 410), new=_ragged(16, 251, 7), heads=16, kv_heads=4, tree=30, window=17, n_sink=5),
    "equal chunks": dict(prefix=_ragged(16, 333, 300), new=[250] * 16, heads=16, kv_heads=4, page=64),
    "chunks under a window": dict(prefix=[300, 2000, 0, 65], new=[999, 1000, 801, 1000], heads=16, kv_heads=4, window=200, n_sink=70),
    "ragged trees under a window": dict(prefix=_ragged(8, 2000), new=[250, 249, 250, 130, 250, 250, 201, 250], heads=32, kv_heads=8, tree=40, window=200, n_sink=2),
    "trees under a window": dict(prefix=_ragged(8, 2000), new=[250] * 7 + [247], heads=32, kv_heads=8, tree=40, window=200),
    "chunks, parts": dict(prefix=[2000, 1777], new=[500, 471], heads=32, kv_heads=8),
    "trees, parts": dict(prefix=[2000, 1777], new=[250, 249], heads=32, kv_heads=8, tree=9),
    "large trees, parts": dict(prefix=[27] + [11] * 14, new=[833] + [416] * 14, heads=4, kv_heads=4, tree=60),
    "long prompts, parts": dict(prefix=[372, 99], new=[3587, 3587], heads=6, kv_heads=2, page=64),
    "trees behind long prefixes": dict(prefix=[33616, 33000], new=[252, 252], heads=32, kv_heads=4, tree=9, page=128),
}

def cut(name, head_dim):
    kw = CASES[name]
    return binding.paged_cut(n_rows=len(kw["prefix"]), n_tokens=sum(kw["new"]), max_new=max(kw["new"]), max_prefix_len=max(kw["prefix"]), n_heads=kw["heads"],
                             n_kv_heads=kw["kv_heads"], head_dim=head_dim, tree="tree" in kw, window=kw.get("window", 0), n_sink=kw.get("n_sink", 0))


def f32_cut(name, head_dim):
    kw = F32[name]
    return binding.paged_cut(n_rows=len(kw["prefix"]), n_tokens=sum(kw["new"]), max_new=max(kw["new"]), max_prefix_len=max(kw["prefix"]), n_heads=kw["heads"],
                             n_kv_heads=kw["kv_heads"], head_dim=head_dim, tree="tree" in kw, window=kw.get("window", 0), dtype=binding.F32)


def _device_attention(q, k, v, sees, scale):
    """As the oracle's attention, on the device: (out, lse, softmax @ |v|, largest sum of |q_d k_d|); values may be infinite or NaN."""
    z = torch.mm(q, k.T.contiguous()) * scale
    z.masked_fill_(~sees, -float("inf"))
    m = z.max(1, keepdim=True).values
    w = torch.exp(z - m)
    total = w.sum(1, keepdim=True)
    fine = torch.where(torch.isfinite(v), v, 0.0)
    out, mag = torch.mm(w, fine) / total, torch.mm(w, fine.abs()) / total
    up, down, nan = (torch.mm(w, x.double()) > 0 for x in (v == float("inf"), v == -float("inf"), torch.isnan(v)))
    out[up], out[down] = float("inf"), -float("inf")
    out[nan | (up & down)] = float("nan")
    size = torch.mm(q.abs(), k.abs().T.contiguous()).mul_(scale).masked_fill_(~sees, 0).max(1).values
    return out, (m + total.log())[:, 0], mag, size


def check(p, kv_heads):
    """As Problem.check, with the non-finite places' values."""
    half, group, odd = 2.0 ** -8, p.heads // p.kv_heads, 0
    for s in range(len(p.prefix)):
        lo, hi = p.off[s], p.off[s + 1]
        if lo == hi:
            continue
        sees = dev(so.visible(p.prefix[s], hi - lo, None if p.parent is None else p.parent[lo:hi], p.window, p.n_sink), bool)
        seen = sees.any(0)                                     # (pages that a window has passed are not there)
        for h in kv_heads:
            k, v = (torch.from_numpy(x).cuda() for x in p.row_keys(s, h))
            k, v = torch.where(seen[:, None], k, 0.0), torch.where(seen[:, None], v, 0.0)
            for g in range(h * group, (h + 1) * group):
                ref, ref_lse, mag, size = _device_attention(p.q[lo:hi, g].double(), k, v, sees, 1 / p.head_dim ** 0.5)
                d = (p.head_dim + 16) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + ref_lse.abs())
                sums = (len(k) + 64) * 2.0 ** -24
                tol = mag * (half + 2 * d[:, None] + sums) + half * ref.abs() + 1e-30
                out = p.out[lo:hi, g].double()
                fine = torch.isfinite(ref)
                odd += int((~fine).sum())
                assert torch.equal(torch.where(fine, 0.0, out.nan_to_num(5.0)), torch.where(fine, 0.0, ref.nan_to_num(5.0))), (s, g, "infinities")
                assert ((out - ref).abs() <= tol)[fine].all(), (s, g, float(((out - ref).abs() / tol)[fine].max()))
                assert ((p.lse[lo:hi, g] - ref_lse).abs() <= 2 * d + sums).all(), (s, g, "lse")
    assert (p.out[p.off[-1]:] == 7).all() and (p.lse[p.off[-1]:] == 7).all()
    return odd


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("name", CASES)
def test_every_cut(name, head_dim):
    kw = dict(CASES[name])
    print(f"[paged cuts] {name} {head_dim} {cut(name, head_dim)}", flush=True)
    p = Problem(list(CASES).index(name), kw.pop("prefix"), kw.pop("new"), head_dim=head_dim, spare=2, **kw)
    heads = sorted({0, p.kv_heads - 1})
    ctx = p.context()
    p.run(ctx)
    assert check(p, heads) == 0
    # infinities and NaN at some keys of every row, one element of the head each
    rng = np.random.default_rng(len(name))
    for s, (prefix, new) in enumerate(zip(p.prefix, p.new)):
        for i, x in enumerate(sorted({0, prefix // 3, max(prefix - 1, 0), prefix, prefix + new // 2, prefix + new - 1, int(rng.integers(0, prefix + new))})):
            if x >= prefix + new:
                continue
            value = (float("inf"), -float("inf"), float("nan"))[(s + i) % 3]
            if x >= prefix:
                p.v_new[p.off[s] + x - prefix, :, 9 * i] = value
            elif p.table[s, x // p.page] < p.k_pages.shape[0]:
                p.v_pages[int(p.table[s, x // p.page]), :, x % p.page, 9 * i] = value
    p.out.fill_(7)
    p.run(ctx)
    assert check(p, heads) > 0
    assert ctx.device_status() == binding.OK


F32 = {
    "one": dict(prefix=[60], new=[3], heads=4, kv_heads=2),
    "parts": dict(prefix=[5000, 3], new=[1, 2], heads=4, kv_heads=1),
    "ranked": dict(prefix=_ragged(8, 500), new=_ragged(8, 200), heads=8, kv_heads=8),
    "ranked, trees, window": dict(prefix=_ragged(8, 500), new=_ragged(8, 200, 1), heads=8, kv_heads=4, tree=20, window=60, n_sink=3),
    "in order": dict(prefix=_ragged(70, 90), new=_ragged(70, 5), heads=8, kv_heads=4),
}


@pytest.mark.parametrize("head_dim", [64, 100, 251])
@pytest.mark.parametrize("name", F32)
def test_every_f32_cut(name, head_dim):
    kw = dict(F32[name])
    print(f"[paged cuts] f32 {name} {head_dim}", flush=True)
    p = Problem(50 + head_dim, kw.pop("prefix"), kw.pop("new"), head_dim=head_dim, dtype="f32", spare=2, **kw)
    ctx = p.context()
    p.run(ctx)
    assert ctx.device_status() == binding.OK
    p.check(sorted({0, p.kv_heads - 1}))
