"""Host-side guard on the compiled kernels of paged_mass and paged_evict (compiles to assembly only: no GPU needed), as for the others over pages: M0 is set by hand for the LDS-direct
loads and nothing else may use it; inline assembly holds only waits, barriers, M0 and those loads."""
import re

import pytest

from test_kernel_registers import LDS_DIRECT, _kernel_stats


@pytest.mark.parametrize("src", ["paged_mass.hip", "paged_evict.hip"])
def test_hand_written_assembly(src, tmp_path):
    stats, text = _kernel_stats(src, tmp_path)
    bodies = re.findall(r"^(_ZN\S*_kernel\S*):[^\n]*\n(.*?)\.amdhsa_kernel", text, flags=re.S | re.M)
    assert len(stats) == len(bodies) > 0
    assert not [(name, spilled) for name, spilled in stats if int(spilled) > 0]
    for name, body in bodies:
        m0 = [l.strip() for l in body.splitlines() if re.search(r"\bm0\b", l)]
        assert all(l.startswith("s_mov_b32 m0,") for l in m0), (name, m0[:5])
        assert bool(m0) == ("global_load_lds_dwordx4" in body) == ("ring_kernel" in name), name
        inline = re.findall(r";;#ASMSTART\n(.*?);;#ASMEND", body, flags=re.S)
        ops = {l.split()[0] for blk in inline for l in blk.strip().splitlines()}
        assert ops <= LDS_DIRECT | {"global_load_lds_dword"}, (name, ops)
