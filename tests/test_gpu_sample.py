"""sample_tokens against the oracle.  Tokens have to be equal: weights are doubles with relative errors below 1e-12, so one uniform in about 1e12 / (entries)
meets a border of the running mass that near (rows of equal weights apart, whose sums are whole numbers on both sides).  A probability is rounded once to
float32."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import serving_oracle as so
from paper_2605_07230_amd import binding

from serving_util import DT, dev

pytestmark = pytest.mark.gpu


def _context(vocab, stream=None):
    return binding.Context(max_rows=1, max_nodes_total=1, max_nodes_per_tree=1, max_prefix=1, n_heads=1, head_dim=64, hidden=64, vocab=vocab, stream=stream)


def _run(logits, u, ctx=None, **par):
    rows = logits.shape[0]
    token, prob = torch.full((rows,), -9, dtype=torch.int32, device="cuda"), torch.full((rows,), -9.0, device="cuda")
    par = {k: dev(v, np.int32 if k == "top_k" else np.float32) for k, v in par.items() if v is not None}
    binding.sample_tokens(ctx or _context(logits.shape[1]), logits=logits, u=dev(u, np.float32), token=token, prob=prob, **par)
    torch.cuda.synchronize()
    return token.cpu().numpy(), prob.cpu().numpy()


def _check(logits, u, **par):
    token, prob = _run(logits, u, **par)
    x = logits.double().cpu().numpy()
    default = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    for r in range(len(x)):
        kw = {k: float(np.float32(par[k][r])) if par.get(k) is not None else v for k, v in default.items()}
        kw["top_k"] = int(kw["top_k"])
        t, p, _ = so.sample(x[r], float(np.float32(u[r])), **kw)
        assert token[r] == t, (r, kw, token[r], t)
        assert abs(prob[r] - p) <= 2.0 ** -23 * p + 1e-12, (r, kw, prob[r], p)


@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 63, 64, 257, 1000, 4096, 4097, 16384, 16385, 33088, 36868, 65533, 65536])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parameters_mixed(vocab, dtype):
    print(f"[sample] {vocab} {dtype}", flush=True)
    rng = np.random.default_rng(vocab)
    rows = 24
    x = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32) * 3).cuda().to(DT[dtype])
    pick = lambda *some: np.array([rng.choice(some) for _ in range(rows)])  # noqa: E731
    _check(x, rng.random(rows) * 0.999, temperature=pick(0, 0.3, 1, 1.7), top_k=pick(0, 1, 40, 2000, 5000, vocab), top_p=pick(1, 0.3, 0.9, 0.99),
           min_p=pick(0, 0, 0.01, 0.2))
    _check(x, rng.random(rows) * 0.999)


@pytest.mark.parametrize("what", ["one value", "two values", "outlier", "masked with the lowest", "masked with -inf", "narrow", "steps", "wide", "all but one masked", "ramp"])
@pytest.mark.parametrize("vocab", [3000, 65536])
def test_rows_that_are_hard_to_cut(what, vocab):
    print(f"[sample] {what} {vocab}", flush=True)
    rng = np.random.default_rng(len(what))
    rows = 12
    x = rng.standard_normal((rows, vocab)).astype(np.float32)
    low = np.finfo(np.float32).min
    if what == "one value":
        x[:] = -3.25
    elif what == "two values":
        x = np.where(rng.random(x.shape) < 0.5, np.float32(1.5), np.float32(-2.5))
    elif what == "outlier":
        x[:, 17] = 3e4
    elif what == "masked with the lowest":
        x[rng.random(x.shape) < 0.99] = low
    elif what == "masked with -inf":
        x[rng.random(x.shape) < 0.9] = -np.inf
    elif what == "narrow":
        x = 100 + x * 1e-4
    elif what == "steps":
        x = np.round(x * 4) / 4
    elif what == "wide":
        x = x * 1e30
    elif what == "all but one masked":
        x[:] = low
        x[np.arange(rows), rng.integers(0, vocab, rows)] = 0.5
    else:
        x[:] = np.linspace(-70, 0, vocab)
    pick = lambda *some: np.array([rng.choice(some) for _ in range(rows)])  # noqa: E731
    x = torch.from_numpy(x.astype(np.float32)).cuda()
    # shares that no sum of equal weights meets exactly
    for par in (dict(), dict(top_k=pick(1, 7, 1500, vocab - 1)), dict(top_p=pick(0.123, 0.6543, 0.98765)), dict(min_p=pick(0.0213, 0.3)),
                dict(top_k=pick(100, 2500), top_p=pick(0.123, 0.6543), min_p=pick(0, 0.0123), temperature=pick(0.5, 1, 2)),
                dict(temperature=pick(1e-6, 1e-3, 50, 1e6), top_p=pick(0.9123, 0.4321)), dict(temperature=pick(0, 1e-6, 1e6), top_k=pick(0, 100))):
        _check(x, rng.random(rows) * 0.999, **par)


def test_edges():
    inf, nan = float("inf"), float("nan")
    rows = torch.tensor([[-inf, nan, -inf, nan], [0, inf, 1, inf], [nan, 0, -inf, 0], [1, 2, 2, 0], [5, 1, 5, 5], [-inf, -inf, 3, -inf]], device="cuda")
    for par in ({}, dict(top_k=[2] * 6), dict(top_p=[0.45] * 6), dict(min_p=[1.0] * 6), dict(temperature=[0.0] * 6), dict(temperature=[inf] * 6, min_p=[1.0] * 6),
                dict(temperature=[0.5] * 6, top_k=[1] * 6, top_p=[0.0] * 6)):
        print(f"[sample] {par}", flush=True)
        for u in (0.0, 0.3, 0.6, 0.999):
            if par.get("temperature", [0])[0] == inf:      # an infinite temperature: all entries above -inf weigh the same
                token, prob = _run(rows[3:4], [u], temperature=[inf], min_p=[1.0])
                assert token[0] == int(u * 4) and prob[0] == 0.25
            else:
                _check(rows, [u] * 6, **par)
    # values that switch a cut off, and uniforms beyond their range
    same = rows[3:5].repeat(2, 1)
    ref = _run(same, [0.7] * 4)
    for par in (dict(top_k=[0, -5, 4, 900]), dict(top_p=[1, nan, 2, inf]), dict(min_p=[0, nan, -1, -inf])):
        got = _run(same, [0.7] * 4, **par)
        assert np.array_equal(got[0], ref[0]) and np.array_equal(got[1], ref[1]), par
    assert _run(same, [1.0, 3.0, inf, 1.0])[0].tolist() == [3, 3, 3, 3] and _run(same, [-1, -inf, nan, 0])[0].tolist() == [0, 0, 0, 0]
    assert _run(same, [0.7] * 4, temperature=[-1, nan, -inf, 0])[0].tolist() == [1, 0, 1, 0]


def test_strides_missing_probabilities_and_streams():
    rng = np.random.default_rng(3)
    wide = torch.from_numpy(rng.standard_normal((9, 1003)).astype(np.float32)).cuda()
    for view in (wide[:, :1000], wide[:, 1:901], wide[::2, 3:1003], torch.cat([wide] * 5, 1)[:, :4100]):
        u = rng.random(view.shape[0]) * 0.999
        _check(view, u, top_k=np.full(view.shape[0], 50))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    token = torch.full((9,), -9, dtype=torch.int32, device="cuda")
    ctx = _context(1003, stream)
    binding.sample_tokens(ctx, logits=wide, u=dev(u[:1].repeat(9), np.float32), token=token)
    stream.synchronize()
    assert token.cpu().tolist() == _run(wide, u[:1].repeat(9))[0].tolist()


def test_many_rows_repeat_bit_for_bit():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = 2 * torch.randn(700, 16384, device="cuda", generator=gen)
    u = torch.rand(700, generator=torch.Generator().manual_seed(2)).numpy()
    par = dict(top_p=np.resize([0.9, 0.5, 1.0], 700), top_k=np.resize([0, 2000], 700), temperature=np.resize([1, 0.7, 1.2, 0.9], 700))
    first = _run(x, u, **par)
    for _ in range(3):
        again = _run(x, u, **par)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])
    _check(x[:20], u[:20], **{k: v[:20] for k, v in par.items()})


def test_refusals():
    E = binding
    x = torch.zeros(2, 64, device="cuda")
    u, token = torch.zeros(2, device="cuda"), torch.full((2,), -9, dtype=torch.int32, device="cuda")
    ctx = _context(64)
    rec = binding._SAMPLE(0, 2, 64, x.data_ptr(), 64, 0, 0, 0, 0, u.data_ptr(), token.data_ptr(), 0)

    def call(**fields):
        a = binding.sample_args.from_buffer_copy(rec)
        for k, v in fields.items():
            setattr(a, k, v)
        return ctx.lib.sample_tokens(ctx.handle, C.byref(a))

    for k in ("logits", "u", "token"):
        assert call(**{k: None}) == E.EINVAL
    assert call(dtype=3) == E.EDTYPE and call(n_rows=-1) == E.EINVAL and call(vocab=0) == E.EINVAL and call(vocab=65) == E.ESHAPE and call(row_stride=63) == E.ESHAPE
    assert ctx.lib.sample_tokens(None, None) == E.EINVAL and call(n_rows=0) == E.OK
    torch.cuda.synchronize()
    assert (token == -9).all()
