"""paged_attn_shared, paged_mass and paged_evict recorded into graphs whose replays overlap with each other and with further calls of their context; calls from other current streams; calls
of several contexts at once; what a call must not touch."""
import pytest
import torch

from paper_2605_07230_amd import binding

from budget_util import Evict, Mass
from test_gpu_paged_shared import make

pytestmark = pytest.mark.gpu


class _Shared:
    def __init__(self, stream, name, workspace):
        self.p = p = make(name, 5)
        self.ctx = p.context(stream)
        self.workspace = None
        if workspace:
            self.workspace = torch.empty(binding.paged_attn_shared_workspace(self.ctx, **p.args, out=p.out), dtype=torch.uint8, device="cuda")
            assert self.workspace.numel() > 0 or name == "few keys"

    def __call__(self):
        binding.paged_attn_shared(self.ctx, **self.p.args, out=self.p.out, lse=self.p.lse, workspace=self.workspace)

    def outputs(self):
        return [self.p.out, self.p.lse]

    def reset(self):
        self.p.out.fill_(7)
        self.p.lse.fill_(7)

    def check(self):
        self.p.check([0, self.p.kv_heads - 1])


class _Mass:
    def __init__(self, stream, seed, new):
        self.p = Mass(seed, [900, 431, 70], [new, 1, 3], heads=8, kv_heads=2, first=[16, 0, 70], path=9)
        self.ctx = self.p.context(stream)

    def __call__(self):
        binding.paged_mass(self.ctx, **self.p.args)

    def outputs(self):
        return [self.p.mass]

    def reset(self):
        self.p.mass.copy_(self.p.before)

    def check(self):
        self.p.check()


class _Evict:
    def __init__(self, stream, seed, recent):
        self.p = Evict(seed, [700, 90, 1500], [400, 80, 900], recent=recent, first=[10, 0, 33])
        self.ctx = self.p.context(stream)
        self.workspace = self.p.workspace(self.ctx)

    def __call__(self):
        binding.paged_evict(self.ctx, **self.p.args, workspace=self.workspace)

    def outputs(self):
        return [self.p.k_pages, self.p.v_pages, self.p.mass_out, *(self.p.args[k] for k in ("free_pages", "seq_len_out", "free_count_out", "dropped"))]

    def reset(self):
        self.p.k_pages.copy_(self.p.was[0])
        self.p.v_pages.copy_(self.p.was[1])
        self.p.mass_out.fill_(-7)
        for k in ("seq_len_out", "free_count_out", "dropped"):
            self.p.args[k].fill_(-9)

    def check(self):
        self.p.check()


def _calls(stream, workspace):
    return [_Shared(stream, "grouped heads", workspace), _Shared(stream, "f32 groups", workspace), _Shared(stream, "few keys", workspace), _Mass(stream, 1, 60), _Mass(stream, 2, 2),
            _Evict(stream, 3, 20), _Evict(stream, 4, 700)]


@pytest.mark.parametrize("workspace", [False, True])
def test_replays_that_overlap(workspace):
    print(f"[budget captured] workspaces {workspace}", flush=True)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        calls, eager = _calls(stream, workspace), []
        for call in calls:
            call()
            eager.append([t.clone() for t in call.outputs()])
            call.check()
    torch.cuda.synchronize()
    graphs, sides = [], []
    for call in calls:
        call.reset()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        sides.append(torch.cuda.Stream())
        with torch.cuda.graph(graphs[-1], stream=stream):
            call()
    with torch.cuda.stream(stream):
        other = _Shared(stream, "not whole tiles", False)                 # what runs beside them, on the same stream as the recorded calls' contexts
    first = None
    for replay in range(6):
        for call in calls:
            call.reset()
        torch.cuda.synchronize()
        for graph, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                graph.replay()
        with torch.cuda.stream(stream):
            for _ in range(3):
                other()
        torch.cuda.synchronize()
        print(f"[budget captured] replay {replay}", flush=True)
        now = [[t.clone() for t in call.outputs()] for call in calls]
        for i, (call, want, got) in enumerate(zip(calls, eager, now)):
            call.check()
            if workspace or i > 2:        # (without one of its own a recorded call takes every row's keys by themselves)
                assert all(torch.equal(a.nan_to_num(-1) if a.is_floating_point() else a, b.nan_to_num(-1) if b.is_floating_point() else b) for a, b in zip(want, got)), i
        other.check()
        first = first or now
        for a, b in zip(first, now):
            assert all(torch.equal(x.nan_to_num(-1) if x.is_floating_point() else x, y.nan_to_num(-1) if y.is_floating_point() else y) for x, y in zip(a, b))
    assert all(call.ctx.device_status() == binding.OK for call in calls)


def test_other_current_streams_and_contexts_at_once():
    """Calls run on their context's stream, whichever is current; contexts on streams of their own do not meet."""
    streams = [torch.cuda.Stream() for _ in range(3)]
    sets = [_calls(s, False) for s in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for calls in sets:
            for call in calls:
                call.reset()
        torch.cuda.synchronize()
        for calls in zip(*sets):
            for call in calls:            # under the default stream
                call()
        torch.cuda.synchronize()
        for calls in sets:
            for call in calls:
                call.check()
                assert call.ctx.device_status() == binding.OK


def test_far_places():
    """Pages beyond 2^31 elements of the pool, tables and weights with long rows."""
    page, kv, d = 64, 4, 128
    pool = (1 << 31) // (kv * page * d) + 40
    big = torch.empty(pool, kv, page, d, dtype=torch.bfloat16, device="cuda")
    last = list(range(pool - 20, pool))
    small = Mass(7, [600, 333], [5, 1], heads=8, kv_heads=kv, page=page)
    ids = [e for e in small.table.reshape(-1).tolist() if e < small.k_pages.shape[0]]
    move = dict(zip(ids, last))
    for a, b in move.items():
        big[b] = small.k_pages[a]
    table = small.args["block_table"].cpu().apply_(lambda e: move.get(e, 1 << 30))
    ctx = small.context()
    wide = torch.full((2, table.shape[1] + 100), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    small.run(ctx, k_pages=big, block_table=wide.cuda()[:, :table.shape[1]])
    assert ctx.device_status() == binding.OK
    small.check()
    p = Evict(8, [600, 333], [300, 200], layers=1, kv_heads=kv, head_dim=d, page=page, recent=9)
    move = {e: last[i] for i, e in enumerate(dict.fromkeys(e for e in p.table.reshape(-1).tolist() if e < p.k_pages.shape[1]))}
    other = torch.empty_like(big)
    for a, b in move.items():
        big[b], other[b] = p.k_pages[0, a], p.v_pages[0, a]
    where = p.args["block_table"].cpu().apply_(lambda e: move.get(e, 1 << 30)).cuda()
    p.run(block_table=where, k_pages=big[None], v_pages=other[None])
    for a, b in move.items():
        p.k_pages[0, a], p.v_pages[0, a] = big[b], other[b]
    back = {b: a for a, b in move.items()}
    p.args["free_pages"].copy_(p.args["free_pages"].cpu().apply_(lambda e: back.get(e, e)))
    p.check()
