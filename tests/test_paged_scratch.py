"""How many registers of a thread the kernels of paged_attn.hip leave in scratch memory (compiles to assembly only: no GPU needed).  Each reload waits for all loads on their way, so the number may
fall but not grow: what is not named here keeps everything in registers."""
from test_kernel_registers import _kernel_stats

# 128-row workgroups of the ring at head_dim 64 (chains, trees): three to a compute unit leave them 168 registers; the other two: trees of few rows at head_dim 64, f32 element by element (by itself, and
# in the kernel of both passes over shared prefixes)
IN_SCRATCH = {"paged_ring_kernelILi64ELi2ELi2ELi4ELb0E": 6, "paged_ring_kernelILi64ELi2ELi2ELi4ELb1E": 4, "paged_few_kernelILi64ELi4ELb1E": 2, "paged_f32_kernelILi4ELi16ELb0E": 2,
              "paged_both_f32_kernelILi4ELi16ELb0E": 2}


def test_registers_in_scratch_memory(tmp_path):
    stats, _ = _kernel_stats("paged_attn.hip", tmp_path)
    for part in IN_SCRATCH:
        assert any(part in name for name, _ in stats), part
    assert not [(name, spilled) for name, spilled in stats if int(spilled) > max((n for part, n in IN_SCRATCH.items() if part in name), default=0)]
