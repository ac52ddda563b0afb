"""Host-side guard on the compiled kernels over pages, as for the step's own (compiles to assembly only: no GPU needed).

M0 is set by hand for the LDS-direct loads and the compiler is not told: nothing else may use it.  Inline assembly is invisible to the
compiler's hazard padding: only waits, barriers, M0 and those loads are written that way."""
import re

import pytest

from test_kernel_registers import LDS_DIRECT, _kernel_stats

WIDE = re.compile(r"paged_ring_kernelILi128E")      # nothing in their tile loops may wait for a reload from scratch


@pytest.mark.parametrize("src", ["paged_attn.hip", "paged_cache.hip", "sample.hip"])
def test_hand_written_assembly(src, tmp_path):
    stats, text = _kernel_stats(src, tmp_path)
    bodies = re.findall(r"^(_ZN\S*_kernel\S*):[^\n]*\n(.*?)\.amdhsa_kernel", text, flags=re.S | re.M)
    assert len(stats) == len(bodies) > 0
    assert not [name for name, spilled in stats if int(spilled) and WIDE.search(name)]
    for name, body in bodies:
        m0 = [l.strip() for l in body.splitlines() if re.search(r"\bm0\b", l)]
        assert all(l.startswith("s_mov_b32 m0,") for l in m0), (name, m0[:5])
        assert bool(m0) == ("global_load_lds_dwordx4" in body) == ("ring_kernel" in name), name
        inline = re.findall(r";;#ASMSTART\n(.*?);;#ASMEND", body, flags=re.S)
        ops = {l.split()[0] for blk in inline for l in blk.strip().splitlines()}
        assert ops <= LDS_DIRECT, (name, ops)
