"""Pages of rows that end, given back as the header says and taken again."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding

from test_gpu_serving_edges import _chunk, _loop

pytestmark = pytest.mark.gpu


def _end(loop, s):
    """Row s ends: its pages lie behind the free ones, its length is 0.  The entry counts come from the device here; a program that counts tokens has them."""
    held, free = -(-int(loop.seq_len[s]) // loop.page_size), int(loop.free_count)
    loop.free_pages[free:free + held] = loop.block_table[s, :held]
    loop.free_count += held
    loop.seq_len[s] = 0


def test_pages_of_a_row_that_ended():
    print("[paged reuse]", flush=True)
    inp, loop = _loop(n_pages=20)                               # 320 positions for two rows of up to 400
    kept = {}
    for turn, (ends, new) in enumerate(((None, [150, 90]), (0, [200, 20]), (1, [3, 60]), (0, [170, 1]))):
        if ends is not None:
            _end(loop, ends)
            kept[ends] = []
        q, k, v = _chunk(inp, sum(new), turn)
        out = torch.empty_like(q)
        loop.admit(q, k, v, new, out)
        torch.cuda.synchronize()
        at = 0
        for s, n in enumerate(new):
            before = kept.setdefault(s, [])
            prefix = sum(len(x[0]) for x in before)
            before.append((k[at:at + n], v[at:at + n]))
            keys, values = (torch.cat([x[i] for x in before]) for i in (0, 1))
            for h in range(inp.n_heads):
                g = h // (inp.n_heads // inp.n_kv_heads)
                ref, _, mag, size = so.attention(q[at:at + n, h].double().cpu().numpy(), keys[:, g].double().cpu().numpy(), values[:, g].double().cpu().numpy(),
                                                 so.visible(prefix, n))
                tol = mag * (2.0 ** -8 + 2 * 80 * 2.0 ** -24 * size[:, None] + 2.0 ** -13) + 2.0 ** -8 * np.abs(ref) + 1e-30
                assert (np.abs(out[at:at + n, h].double().cpu().numpy() - ref) <= tol).all(), (turn, s, h)
            at += n
            pages = loop.block_table[s, :-(-len(keys) // loop.page_size)].long()
            for pool, rows in ((loop.k_pages, keys), (loop.v_pages, values)):
                assert torch.equal(pool[0, pages].transpose(1, 2).reshape(-1, inp.n_kv_heads, inp.head_dim)[:len(rows)], rows), (turn, s)
        held = torch.cat([loop.block_table[s, :-(-int(loop.seq_len[s]) // loop.page_size)] for s in range(2)])
        free = loop.free_pages[:int(loop.free_count)]
        assert sorted(torch.cat([held, free]).tolist()) == list(range(20))        # every page is held once, or free
        assert loop.ctx.device_status() == binding.OK
