"""What the calls on pages and draws allow beyond ordinary use: places further apart than 32 bits count, contexts at work at once, a current stream that is not the context's."""
import numpy as np
import pytest
import torch

from paper_2605_07230_amd import binding
from paper_2605_07230_amd import decode
from paper_2605_07230_amd import workloads as wl

from serving_util import Problem, dev

pytestmark = pytest.mark.gpu

# one for every way a call is cut: 16 and 32 query rows, 64 / 128 / 256 of them, f32
SHAPES = {
    "tokens": dict(prefix=[50, 77], new=[1, 1], heads=4, kv_heads=2),
    "few": dict(prefix=[50, 77], new=[5, 8], heads=8, kv_heads=2),
    "64": dict(prefix=[50, 77], new=[40, 33], heads=2, kv_heads=2),
    "128": dict(prefix=[50, 77], new=[120, 90], heads=2, kv_heads=2),
    "256": dict(prefix=[90], new=[300], heads=8, kv_heads=2, head_dim=64),
    "tree": dict(prefix=[50, 77], new=[60, 200], heads=4, kv_heads=2, tree=7),
    "window": dict(prefix=[150, 77], new=[100, 20], heads=4, kv_heads=2, window=60, n_sink=2),
    "f32": dict(prefix=[50, 77], new=[40, 1], heads=4, kv_heads=2, dtype="f32", head_dim=72),
    "f32 odd": dict(prefix=[50, 77], new=[4, 1], heads=4, kv_heads=2, dtype="f32", head_dim=67),
}


def _apart(t, step):
    """The same values with the first dimension's elements `step` elements apart."""
    inner = t.contiguous()
    big = torch.empty((t.shape[0] - 1) * step + inner[0].numel(), dtype=t.dtype, device=t.device)
    far = big.as_strided(t.shape, (step, *inner.stride()[1:]))
    far.copy_(t)
    return far


@pytest.mark.parametrize("name", SHAPES)
def test_pages_past_32_bits(name):
    kw = dict(SHAPES[name])
    print(f"[serving edges] pages {name}", flush=True)
    p = Problem(3, kw.pop("prefix"), kw.pop("new"), **kw)
    p.run()
    p.check()
    out, lse = p.out.clone(), p.lse.clone()
    n = p.k_pages.shape[0]
    step = (5 << 30) // (n - 1) // p.k_pages.element_size() & ~7           # 5 GB from the first page to the last
    p.out.fill_(7)
    p.run(k_pages=_apart(p.k_pages, step), v_pages=_apart(p.v_pages, step))
    assert torch.equal(p.out, out) and torch.equal(p.lse, lse)


@pytest.mark.parametrize("name", SHAPES)
def test_tokens_past_32_bits(name):
    kw = dict(SHAPES[name])
    print(f"[serving edges] tokens {name}", flush=True)
    p = Problem(4, kw.pop("prefix"), kw.pop("new"), **kw)
    p.run()
    p.check()
    out, lse = p.out.clone(), p.lse.clone()
    step = min((5 << 30) // max(p.n - 1, 1) // p.q.element_size(), 1 << 25) & ~7      # 5 GB from the first token to the last, where kv_stride may be so large
    p.out.fill_(7)
    p.run(q=_apart(p.q, step), k_new=_apart(p.k_new, step), v_new=_apart(p.v_new, step))
    assert torch.equal(p.out, out) and torch.equal(p.lse, lse)


@pytest.mark.parametrize("name", ["tokens", "64", "256", "f32"])
def test_positions_far_apart(name):
    """The largest step from one position of a page to the next."""
    kw = dict(SHAPES[name])
    print(f"[serving edges] positions {name}", flush=True)
    p = Problem(5, kw.pop("prefix"), kw.pop("new"), **kw)
    p.run()
    out, lse = p.out.clone(), p.lse.clone()
    far = [_apart(x.permute(2, 0, 1, 3), 1 << 25).permute(1, 2, 0, 3) for x in (p.k_pages, p.v_pages)]
    p.out.fill_(7)
    p.run(k_pages=far[0], v_pages=far[1])
    assert torch.equal(p.out, out) and torch.equal(p.lse, lse)
    p.check()


def test_rows_of_logits_far_apart():
    print("[serving edges] logits", flush=True)
    x = (2 * torch.randn(3, 5000, device="cuda")).bfloat16()
    far = _apart(x, (3 << 29) + 8)
    ctx = binding.Context(max_rows=1, max_nodes_total=1, max_nodes_per_tree=1, max_prefix=1, n_heads=1, head_dim=64, hidden=64, vocab=5000)
    got = []
    for logits in (x, far):
        token, prob = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
        binding.sample_tokens(ctx, logits=logits, u=dev([0.1, 0.6, 0.9], np.float32), token=token, prob=prob, top_p=dev([0.9, 1.0, 0.5], np.float32), top_k=dev([0, 20, 0]))
        got.append((token, prob))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_two_contexts_at_once():
    """Two programs of one process, a context and a stream each, whose calls cut their keys into parts."""
    print("[serving edges] two contexts", flush=True)
    streams = [torch.cuda.Stream() for _ in range(2)]
    problems = [Problem(20 + i, [3000 - 500 * i, 900], [1, 1 + i], heads=16, kv_heads=4, page=32) for i in range(2)]
    contexts = [p.context(s) for p, s in zip(problems, streams)]
    first = None
    for turn in range(10):
        for p in problems:
            p.out.fill_(7)
        torch.cuda.synchronize()
        for _ in range(5):
            for p, ctx in zip(problems, contexts):
                binding.paged_attn(ctx, **p.args, out=p.out, lse=p.lse)
        torch.cuda.synchronize()
        for p in problems:
            p.check()
        now = [(p.out.clone(), p.lse.clone()) for p in problems]
        first = first or now
        assert all(torch.equal(a, b) for x, y in zip(first, now) for a, b in zip(x, y))


def _loop(**kw):
    inp = wl.make_inputs(name="serving_edges", seed=3, dtype="bf16", n_prompts=2, cfg=False, n_heads=4, n_kv_heads=2, head_dim=64, hidden=128, vocab=1024,
                         prefix_lens=[100, 60], trees=[wl.grow_tree(np.random.default_rng(1), n, 4, 6) for n in (20, 30)], cfg_scale=3.0, temperature=1.0, top_k=100,
                         tau_pos=0.8, tau_seq=0.5, eps_tvd=0.5, token_law="zipf")
    return inp, decode.PagedLoop(inp, page_size=16, max_len=400, max_chunk=128, **kw)


def _chunk(inp, n, seed=1):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return [torch.randn(n, h, inp.head_dim, device="cuda", generator=gen).bfloat16() for h in (inp.n_heads, inp.n_kv_heads, inp.n_kv_heads)]


def test_the_loop_refuses_chunks_before_it_gives_pages():
    print("[serving edges] refused chunks", flush=True)
    inp, loop = _loop()
    for n, new in ((300, [150, 150]), (20, [20]), (20, [15, 15]), (20, [-1, 5])):
        q, k, v = _chunk(inp, n)
        with pytest.raises(ValueError):
            loop.admit(q, k, v, new, torch.empty_like(q))
    assert loop.seq_len.tolist() == [0, 0] and int(loop.free_count) == loop.n_pages and loop.longest == 0
    q, k, v = _chunk(inp, 20)
    out = torch.full_like(q, 7)
    loop.admit(q, k, v, [0, 0], out)
    torch.cuda.synchronize()
    assert (out == 7).all() and loop.seq_len.tolist() == [0, 0]
    loop.admit(q, k, v, [0, 15], out)                      # five tokens behind the last row
    torch.cuda.synchronize()
    assert (out[15:] == 7).all() and loop.seq_len.tolist() == [0, 15] and loop.ctx.device_status() == binding.OK


def test_the_loop_under_another_current_stream():
    print("[serving edges] current stream", flush=True)
    results = []
    for other in (False, True):
        inp, loop = _loop()
        q, k, v = _chunk(inp, 160)
        out = torch.empty_like(q)
        u, token = dev([0.3, 0.8], np.float32), torch.empty(2, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream() if other else torch.cuda.current_stream()):
            loop.admit(q, k, v, [100, 60], out)
            for _ in range(3):
                loop.step()
            loop.draw(u, token)
        torch.cuda.synchronize()
        assert loop.ctx.device_status() == binding.OK
        results.append((out, loop.step_in.attn_out, loop.seq_len, loop.block_table, token))
    assert all(torch.equal(a, b) for a, b in zip(*results))
