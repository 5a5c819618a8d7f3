"""Registers of the kernels for new tokens and their logits, from the notes in the library's code objects."""
import re

from tests.test_registers import workgroups
from tests.test_tree_registers import of


def test_the_passes_spill_nothing():
    """Two wavefronts share a SIMD's registers in the bf16 kernels, also where one kernel has tiles of 256 rows and requests of few rows."""
    for name, k in of("prompt_pass").items():
        assert k[".vgpr_spill_count"] == 0, (name, k[".vgpr_count"], k[".vgpr_spill_count"])
        if re.search(r"CfgILi\d+ELi\d+ELb0E", name):
            assert workgroups(k) >= 2, (name, k[".vgpr_count"])
    for name, k in of("prompt_merge").items():
        assert k[".vgpr_spill_count"] == 0, name


def test_scans_of_logits_leave_room_for_five_wavefronts():
    for name, k in of("logprob_pass").items():
        assert k[".vgpr_spill_count"] == 0 and workgroups(k) >= 5, (name, k[".vgpr_count"])
