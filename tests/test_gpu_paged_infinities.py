"""Infinities and NaN among values that tokens attend, over pages: such a token's output holds that infinity (or NaN) and nothing else, wherever the key lies - in the first
tile of a row or of a part, as the last cached key, as a single token's own - and every other output is exact."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding

from serving_util import Problem

pytestmark = pytest.mark.gpu

SHAPES = {
    "tokens": dict(prefix=[40, 64, 0, 65], new=[1, 1, 1, 1]),
    "tokens, narrow": dict(prefix=[40, 64, 0, 65], new=[1, 1, 1, 1], head_dim=64),
    "tokens, parts": dict(prefix=[3001, 90], new=[1, 1]),
    "tokens, window": dict(prefix=[400, 90], new=[1, 1], window=33, n_sink=2),
    "few": dict(prefix=[40, 70], new=[5, 8]),
    "few, tree": dict(prefix=[40, 70], new=[5, 8], tree=3),
    "prompts": dict(prefix=[0, 0], new=[100, 33]),
    "prompts, narrow": dict(prefix=[0, 0], new=[100, 33], head_dim=64),
    "chunks": dict(prefix=[100, 130], new=[100, 33]),
    "chunks, parts": dict(prefix=[6001], new=[40], kv_heads=1),
    "chunks, window": dict(prefix=[100, 30], new=[100, 40], window=50, n_sink=3),
    "trees": dict(prefix=[100, 0], new=[100, 33], tree=6),
    "trees, window, narrow": dict(prefix=[100, 20], new=[100, 33], tree=9, window=5, n_sink=6, head_dim=64),
    "f32": dict(prefix=[40, 0], new=[1, 40], dtype="f32", head_dim=72),
    "f32, tree": dict(prefix=[40, 0], new=[3, 40], dtype="f32", head_dim=64, tree=5),
}


def _put(p, s, x, d, value):
    """`value` at place x of row s (cached, then new), all kv heads, element d."""
    if x >= p.prefix[s]:
        p.v_new[p.off[s] + x - p.prefix[s], :, d] = value
    elif p.table[s, x // p.page] < p.k_pages.shape[0]:            # (a page that a window has passed is not there)
        p.v_pages[int(p.table[s, x // p.page]), :, x % p.page, d] = value


def _check_all(p):
    p.check()                                                     # which places are finite, and what stands in them
    out = p.out.double().cpu().numpy()
    seen = 0
    for s in range(len(p.prefix)):
        lo, hi = p.off[s], p.off[s + 1]
        sees = so.visible(p.prefix[s], hi - lo, None if p.parent is None else p.parent[lo:hi], p.window, p.n_sink)
        for g in range(p.heads):
            k, v = p.row_keys(s, g // (p.heads // p.kv_heads))
            ref = so.attention(p.q[lo:hi, g].double().cpu().numpy(), k, v, sees)[0]
            other = ~np.isfinite(ref)
            seen += other.sum()
            assert np.array_equal(out[lo:hi, g][other], ref[other], equal_nan=True), (s, g, out[lo:hi, g][other][:5], ref[other][:5])
    return seen


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.filterwarnings("ignore:invalid value")
def test_values_that_a_token_attends(name):
    kw = dict(SHAPES[name])
    for place in ("first new", "last new", "first cached", "last cached", "several"):
        print(f"[paged infinities] {name}: {place}", flush=True)
        p = Problem(31, kw["prefix"], kw["new"], **{"heads": 4, "kv_heads": 2, **{k: v for k, v in kw.items() if k not in ("prefix", "new")}})
        for s, (prefix, new) in enumerate(zip(p.prefix, p.new)):
            at = {"first new": [prefix], "last new": [prefix + new - 1], "first cached": [0], "last cached": [max(prefix - 1, 0)],
                  "several": [0, prefix // 2, prefix, prefix + new // 2]}[place]
            for i, x in enumerate(at):
                _put(p, s, x, 5 + 16 * i, float("inf"))
                _put(p, s, x, 6 + 16 * i, -float("inf"))
                _put(p, s, x, 7 + 16 * i, float("nan"))
        ctx = p.context()
        p.run(ctx)
        assert ctx.device_status() == binding.OK
        assert _check_all(p) > 0 or "window" in name
