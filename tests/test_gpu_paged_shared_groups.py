"""Groups of paged_attn_shared that are out of order are reported whatever way the call takes: calls that paged_attn takes alone, too few to share, recorded ones, of every kernel."""
import pytest
import torch

from paper_2605_07230_amd import binding

from serving_util import dev
from test_gpu_paged_shared import ALONE, make, rows, some_heads, Shared

pytestmark = pytest.mark.gpu

NAMES = [n for n in ALONE if len(ALONE[n]["groups"]) >= 2]


def bad_offsets(n_groups, n_rows):
    """Every way to be out of order, with n_groups groups."""
    good = [min(g, n_rows) for g in range(n_groups)] + [n_rows]
    yield [1, *good[1:]]
    yield [-1, *good[1:]]
    yield [*good[:-1], n_rows - 1]
    yield [*good[:-1], n_rows + 1]
    if n_groups > 1:
        yield [0, n_rows, *[n_rows - 1] * (n_groups - 2), n_rows] if n_groups > 2 else [0, n_rows + 1, n_rows]
        yield [0, -1 << 31, *good[2:]]


@pytest.mark.parametrize("name", NAMES)
def test_calls_that_share_nothing(name):
    p = make(name, 40)
    n = len(p.shared)
    assert p.cut()[1] == 0
    p.run()
    for groups in bad_offsets(n, len(p.prefix)):
        print(f"[paged_attn_shared] {name}: {groups}", flush=True)
        ctx = p.context()
        want = p.out.clone(), p.lse.clone()
        p.out.fill_(7), p.lse.fill_(7)
        p.run(ctx, group_off=dev(groups))
        assert ctx.device_status() == binding.ETREE, groups
        assert torch.equal(p.out, want[0]) and torch.equal(p.lse, want[1])
        p.run(ctx)                                                  # in order again: nothing to report
        assert ctx.device_status() == binding.OK
    p.check(some_heads(p))


def test_more_offsets_than_threads_look_at_once():
    """A thousand empty groups in front of the rows, the last offset but one out of order."""
    p = Shared(41, [70, 80], [1, 1], [0, 2], [0], heads=4, kv_heads=2)
    shared = dev([0] * 1001)
    for groups, status in (([0] * 1000 + [0, 2], binding.OK), ([0] * 1000 + [3, 2], binding.ETREE), ([0] * 400 + [1] + [0] * 600 + [2], binding.ETREE)):
        ctx = p.context()
        p.run(ctx, group_off=dev(groups), shared_len=shared)
        assert ctx.device_status() == status
        p.check(some_heads(p))


def test_recorded_without_a_workspace():
    """Such a call shares nothing; its groups are looked at in every replay."""
    p = Shared(42, rows(16, 1040, 1050), rows(16, 1), [0, 16], [1040], heads=32, kv_heads=32)
    stream = torch.cuda.Stream()
    groups = dev([0, 16])
    with torch.cuda.stream(stream):
        ctx = p.context(stream=stream)
        args = {**p.args, "out": p.out, "lse": p.lse, "group_off": groups}
        binding.paged_attn_shared(ctx, **args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.paged_attn_shared(ctx, **args)
    for last, status in ((16, binding.OK), (15, binding.ETREE), (16, binding.OK), (17, binding.ETREE)):
        groups.copy_(dev([0, last]))
        p.out.fill_(7)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        assert ctx.device_status() == status, last
        p.check(some_heads(p))
