"""Prompts, verification steps, commits and draws over pages, chained as a serving program chains them, against the same steps on a contiguous cache."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding
from paper_2605_07230_amd import decode
from paper_2605_07230_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _inputs(dtype, cfg):
    rng = np.random.default_rng(5)
    return wl.make_inputs(name="paged_loop", seed=11, dtype=dtype, n_prompts=3, cfg=cfg, n_heads=8, n_kv_heads=2, head_dim=64, hidden=256, vocab=4096,
                          prefix_lens=[p for p in (170, 33, 400) for _ in range(2 if cfg else 1)], trees=[wl.grow_tree(rng, n, 6, 8) for n in (40, 21, 60)], cfg_scale=3.0, temperature=1.0, top_k=200,
                          tau_pos=0.8, tau_seq=0.5, eps_tvd=0.5, token_law="zipf")


@pytest.mark.parametrize("dtype,cfg", [("bf16", True), ("bf16", False), ("f32", True)])
def test_steps_over_pages_equal_steps_over_a_contiguous_cache(dtype, cfg):
    inp = _inputs(dtype, cfg)
    print(f"[paged loop] {dtype} guidance {cfg}", flush=True)
    plain = binding.DeviceStep(inp)
    S, steps, cap = inp.n_rows, 3, 640
    k_cache = torch.zeros(1, S, inp.n_kv_heads, cap, inp.head_dim, dtype=plain.q.dtype, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    k_cache[0, :, :, :inp.prefix_cap], v_cache[0, :, :, :inp.prefix_cap] = plain.k_cache, plain.v_cache
    prefix, nxt = plain.prefix_len.clone(), torch.empty_like(plain.prefix_len)
    ctx = binding.Context(max_rows=S, max_nodes_total=inp.q.shape[0], max_nodes_per_tree=plain.max_tree, max_prefix=cap, n_heads=inp.n_heads,
                          head_dim=inp.head_dim, hidden=inp.hidden, vocab=inp.vocab)

    loop = decode.PagedLoop(inp, page_size=16, max_len=cap, max_chunk=400, n_pages=S * 40 + 3)
    # the prompts arrive in two chunks; their attention is checked against the oracle
    done = np.zeros(S, np.int64)
    for part in range(2):
        new = [int(p) // 2 if part == 0 else int(p) - int(p) // 2 for p in inp.prefix_len]
        rows = [(s, int(done[s]), int(done[s]) + new[s]) for s in range(S)]
        k_new = torch.cat([k_cache[0, s, :, a:b].transpose(0, 1) for s, a, b in rows]).contiguous()
        v_new = torch.cat([v_cache[0, s, :, a:b].transpose(0, 1) for s, a, b in rows]).contiguous()
        q = torch.randn(k_new.shape[0], inp.n_heads, inp.head_dim, device="cuda").to(k_new.dtype)
        out = torch.empty_like(q)
        loop.admit(q, k_new, v_new, new, out)
        torch.cuda.synchronize()
        at = 0
        for s, a, b in rows:
            for h in (0, 5):
                kk, vv = (x[0, s, h // 4, :b].double().cpu().numpy() for x in (k_cache, v_cache))
                ref, _, mag, size = so.attention(q[at:at + b - a, h].double().cpu().numpy(), kk, vv, so.visible(a, b - a))
                tol = mag * ((2 * 2.0 ** -8 if dtype == "bf16" else 0) + 2 * 96 * 2.0 ** -24 * size[:, None] + 600 * 2.0 ** -24) + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0)
                assert (np.abs(out[at:at + b - a, h].double().cpu().numpy() - ref) <= tol + 1e-30).all(), (s, h)
            at += b - a
        done += new
    assert torch.equal(loop.seq_len, prefix)

    def same_cache():
        for s in range(S):
            n = int(prefix[s])
            pages = loop.block_table[s, :-(-n // 16)].long()
            for pool, cache in ((loop.k_pages, k_cache), (loop.v_pages, v_cache)):
                got = pool[0, pages].transpose(1, 2).reshape(-1, inp.n_kv_heads, inp.head_dim)[:n]
                assert torch.equal(got, cache[0, s, :, :n].transpose(0, 1)), s
        held = torch.cat([loop.block_table[s, :-(-int(prefix[s]) // 16)] for s in range(S)])
        assert held.unique().numel() == held.numel() == loop.n_pages - int(loop.free_count)

    same_cache()
    for step in range(steps):
        binding.tree_verify_attn(ctx, node_off=plain.row_node_off, parent=plain.row_parent, prefix_len=prefix, q=plain.q, k_tree=plain.k_tree, v_tree=plain.v_tree,
                                 k_cache=k_cache[0], v_cache=v_cache[0], out=plain.attn_out, lse=plain.attn_lse, max_nodes_per_tree=plain.max_tree, max_prefix_len=cap)
        plain.lmhead()
        plain.accept()
        plain.select()
        binding.kv_commit(ctx, node_off=plain.row_node_off, row_prompt=loop.row_prompt, accept_len=plain.accept_len, path_nodes=plain.path_nodes,
                          k_tree=plain.k_tree.unsqueeze(0), v_tree=plain.v_tree.unsqueeze(0), k_cache=k_cache, v_cache=v_cache, prefix_len=prefix, prefix_len_out=nxt)
        prefix, nxt = nxt, prefix
        loop.step()
        torch.cuda.synchronize()
        st = loop.step_in
        for k in ("accept_len", "path_nodes", "emitted", "terminal"):
            assert torch.equal(getattr(st, k), getattr(plain, k)), k
        # both within what a rounded probability and a rounded result leave of the values' size (below 6 for these)
        tol = 4 * 2.0 ** -8 * 6 if dtype == "bf16" else 1e-5
        assert (st.attn_out.float() - plain.attn_out.float()).abs().max() <= tol and (st.attn_lse - plain.attn_lse).abs().max() <= 1e-2
        assert torch.equal(loop.seq_len, prefix)
        same_cache()
    # plain decoding: a token of every prompt from its root's logits
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    token, prob = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    par = dict(temperature=[1.0, 0.7, 0.0], top_k=[50, 0, 0], top_p=[1.0, 0.9, 1.0])
    loop.draw(u, token, prob, **{k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in par.items()})
    for b in range(3):
        want = so.sample(loop.step_in.logits[int(inp.node_off[b])].double().cpu().numpy(), float(u[b]), par["temperature"][b], par["top_k"][b],
                         float(np.float32(par["top_p"][b])))
        assert int(token[b]) == want[0] and abs(float(prob[b]) - want[1]) <= 2.0 ** -23
    assert loop.ctx.device_status() == binding.OK


def test_rows_without_pages_stay_as_they_are():
    inp = _inputs("bf16", False)
    loop = decode.PagedLoop(inp, page_size=64, max_len=640, max_chunk=400, n_pages=9)      # the prompts ask for 3 + 1 + 7 pages
    new = [int(p) for p in inp.prefix_len]
    n = sum(new)
    mk = lambda h: torch.randn(n, h, inp.head_dim, device="cuda").bfloat16()  # noqa: E731
    q = mk(inp.n_heads)
    loop.admit(q, mk(inp.n_kv_heads), mk(inp.n_kv_heads), new, torch.empty_like(q))
    assert loop.ctx.device_status() == binding.ETREE
    assert loop.seq_len.tolist() == [new[0], new[1], 0] and int(loop.free_count) == 5
