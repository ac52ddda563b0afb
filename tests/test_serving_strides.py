"""Views of paged_attn's tensors whose strides say nothing: no GPU needed, nothing is launched."""
import pytest
import torch

from paper_2605_07230_amd import binding as B


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_strides_of_single_tokens_and_single_heads():
    """A dimension of one element has any stride: what comes out of a transposition is taken like what was made in place."""
    def record(q, k, v):
        return B.paged_attn_args.from_buffer_copy(B._paged_attn_record(_i32(2), _i32(1), _i32(1, 4), q, k, v, _bf16(9, k.shape[1], 16, 64), _bf16(9, k.shape[1], 16, 64),
                                                                       torch.empty(q.shape, dtype=q.dtype), None, None, 0.0, 0, 0, 1, 0, None))
    one = record(_bf16(8, 1, 64).transpose(0, 1), _bf16(2, 1, 64).transpose(0, 1), _bf16(2, 1, 64).transpose(0, 1))
    assert one.q_stride == 8 * 64 and one.kv_stride == 2 * 64 and one.n_tokens == 1
    shared = record(_bf16(5, 8, 64), _bf16(1, 5, 64).transpose(0, 1), _bf16(1, 5, 64).transpose(0, 1))
    assert shared.kv_stride == 64 and shared.n_kv_heads == 1 and shared.n_tokens == 5
    wide = _bf16(5, 10, 64)
    assert record(wide[:, :8], wide[:, 8:9], wide[:, 9:]).kv_stride == 640
    alone = record(_bf16(1, 5, 64).transpose(0, 1), _bf16(1, 5, 64).transpose(0, 1), _bf16(1, 5, 64).transpose(0, 1))
    assert alone.q_stride == 64 and alone.kv_stride == 64
    with pytest.raises(AssertionError):                                     # heads that do not lie behind each other
        record(_bf16(8, 5, 64).transpose(0, 1), _bf16(5, 2, 64), _bf16(5, 2, 64))
