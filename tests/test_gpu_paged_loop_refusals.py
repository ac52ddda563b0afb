"""What PagedLoop.admit refuses leaves lengths, tables and pages as they were."""
import pytest
import torch

from paper_2605_07230_amd import binding

from test_gpu_serving_edges import _chunk, _loop

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["slices of one projection", "values in f32", "keys of another number", "out apart", "out of another size", "queries off their boundary"])
def test_refused_tensors_leave_the_loop_as_it_was(what):
    print(f"[paged loop] refused: {what}", flush=True)
    inp, loop = _loop()
    new = [20, 10]
    q, k, v = _chunk(inp, 30)
    out = torch.full_like(q, 7)
    good = q, k, v, out
    if what == "slices of one projection":
        kv = torch.cat([k, v], 1)
        k, v = kv[:, :inp.n_kv_heads], kv[:, inp.n_kv_heads:]
    elif what == "values in f32":
        v = v.float()
    elif what == "keys of another number":
        k = k[:29]
    elif what == "out apart":
        out = torch.full((30, 2 * inp.n_heads, inp.head_dim), 7.0, device="cuda", dtype=q.dtype)[:, :inp.n_heads]
    elif what == "out of another size":
        out = out[:29]
    else:
        q = torch.cat([q.flatten()[:1], q.flatten()])[1:].view(q.shape)
    with pytest.raises((AssertionError, binding.CascadeError)):
        loop.admit(q, k, v, new, out)
    torch.cuda.synchronize()
    assert loop.seq_len.tolist() == [0, 0] and int(loop.free_count) == loop.n_pages and loop.longest == 0 and (out == 7).all()
    assert (loop.k_pages == 0).all() and (loop.v_pages == 0).all()
    q, k, v, out = good
    loop.admit(q, k, v, new, out)
    torch.cuda.synchronize()
    assert loop.seq_len.tolist() == new and loop.ctx.device_status() == binding.OK
    assert torch.equal(loop.k_pages[0, int(loop.block_table[0, 0]), :, 3], k[3])
