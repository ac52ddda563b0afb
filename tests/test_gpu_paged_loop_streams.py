"""Tensors that PagedLoop is given under another current stream: their memory may not be handed out on that stream before the loop's own has read it."""
import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding

from serving_util import dev
from test_gpu_serving_edges import _chunk, _loop

pytestmark = pytest.mark.gpu


def _span(t):
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


def _meet(a, b):
    return any(x[0] < y[1] and y[0] < x[1] for x in a for y in b)


@pytest.mark.parametrize("what", ["admit", "draw"])
def test_given_tensors_stay_until_they_are_read(what, monkeypatch):
    print(f"[paged loop] tensors of another stream: {what}", flush=True)
    inp, loop = _loop()
    loop.step()                                                  # logits for the draw
    busy = torch.randn(8192, 8192, device="cuda")
    slots = binding.paged_slots

    def late(*args, **kw):                                       # behind the copy of the lengths, which waits: some 150 ms on the loop's stream
        for _ in range(20):
            torch.mm(busy, busy)
        slots(*args, **kw)

    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        if what == "admit":
            q, k, v = _chunk(inp, 160)
            given = [q, k, v, torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")]
            del q, k, v
        else:
            given = [dev([0.3, 0.8], np.float32), dev([7, 7]), torch.empty(2, device="cuda"), dev([0.9, 0.5], np.float32), dev([0, 40])]
        torch.cuda.synchronize()
        monkeypatch.setattr(binding, "paged_slots", late)
        if what == "admit":
            loop.admit(*given[:3], [100, 60], *given[3:])
        else:
            loop._place(2, new_len=torch.zeros_like(loop.seq_len))
            loop.draw(*given[:3], top_p=given[3], top_k=given[4])
        spans = [_span(t) for t in given]
        shapes = [(t.shape, t.dtype) for t in given]
        del given
        again = [torch.empty(s, dtype=d, device="cuda") for s, d in shapes]
        assert not loop.ctx.stream.query()                       # the loop's stream has not come to them
        assert not _meet(spans, [_span(t) for t in again])
    torch.cuda.synchronize()
    assert loop.ctx.device_status() == binding.OK


def test_every_call_of_a_step_is_made_on_the_loops_stream_and_device(monkeypatch):
    """The step's older calls launch on the device that is current: the loop makes its own current, whichever one the caller left."""
    print("[paged loop] calls of a step", flush=True)
    _, loop = _loop()
    seen = []

    def watched(owner, name):
        call = getattr(owner, name)

        def watch(*args, **kw):
            seen.append((name, torch.cuda.current_stream(), torch.cuda.current_device()))
            return call(*args, **kw)

        monkeypatch.setattr(owner, name, watch)

    for name in ("lmhead", "accept", "select"):
        watched(loop.step_in, name)
    for name in ("paged_attn", "paged_slots", "paged_append"):
        watched(binding, name)
    with torch.cuda.stream(torch.cuda.Stream()):
        loop.step()
    torch.cuda.synchronize()
    assert [x[0] for x in seen] == ["paged_attn", "lmhead", "accept", "select", "paged_slots", "paged_append"]
    assert all(x[1:] == (loop.ctx.stream, loop.dev.index) for x in seen)
    assert loop.ctx.device_status() == binding.OK
