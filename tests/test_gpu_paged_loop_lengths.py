"""PagedLoop rows that grow into the last page of their table, where max_len is no multiple of the page size."""
import pytest
import torch

from paper_2605_07230_amd import binding
from paper_2605_07230_amd import decode

from test_gpu_serving_edges import _chunk, _loop

pytestmark = pytest.mark.gpu


def _grown(max_len):
    inp, _ = _loop()
    loop = decode.PagedLoop(inp, page_size=64, max_len=max_len, max_chunk=400)
    results = []
    for seed, new in enumerate(([390, 60], [40, 1])):            # 430 positions: past 400, inside the seventh page
        q, k, v = _chunk(inp, sum(new), seed)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        loop.admit(q, k, v, new, out, lse)
        results += [out, lse]
    for _ in range(2):
        loop.step()
        results += [loop.step_in.attn_out.clone(), loop.step_in.attn_lse.clone(), loop.seq_len.clone()]
    torch.cuda.synchronize()
    return loop, results


def test_a_row_past_max_len_in_its_last_page():
    print("[paged loop] 400 positions in pages of 64", flush=True)
    loop, got = _grown(400)
    assert loop.ctx.device_status() == binding.OK
    _, want = _grown(448)
    assert int(got[-1][0]) > 430 and all(torch.isfinite(x).all() for x in got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_row_stays_where_its_table_ends():
    print("[paged loop] a full table", flush=True)
    loop, _ = _grown(400)
    before = loop.seq_len.tolist()
    inp = loop.inp
    q, k, v = _chunk(inp, 100)
    loop.admit(q, k, v, [60, 40], torch.empty_like(q))
    assert loop.seq_len.tolist() == [before[0], before[1] + 40] and loop.ctx.device_status() == binding.ETREE
    loop.step()                                                  # and is attended as it is
    assert torch.isfinite(loop.step_in.attn_lse).all() and loop.ctx.device_status() in (binding.OK, binding.ETREE)
