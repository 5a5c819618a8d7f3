"""Registers of the kernels for trees and eviction, from the notes in the library's code objects."""
import re

from tests.test_registers import kernels, workgroups


def of(name):
    found = {n: k for n, k in kernels().items() if re.search(rf"\d{name}I", n)}
    assert found, f"no {name}"
    return found


def test_the_pass_spills_nothing():
    """Two wavefronts share a SIMD's registers in the bf16 kernels; a spilled register is fetched anew for every tile (92 of them took the pass
    over 64 fp8 requests from 446 to 949 us)."""
    for name, k in of("tree_pass").items():
        assert k[".vgpr_spill_count"] == 0, (name, k[".vgpr_count"], k[".vgpr_spill_count"])
        if re.search(r"CfgILi\d+ELi\d+ELb0E", name):
            assert workgroups(k) >= 2, (name, k[".vgpr_count"])


def test_the_statistic_and_the_merge_spill_nothing():
    for kernel in ("tree_scores", "tree_merge"):
        for name, k in of(kernel).items():
            assert k[".vgpr_spill_count"] == 0, (name, k[".vgpr_count"], k[".vgpr_spill_count"])


def test_two_workgroups_of_a_selection_share_a_compute_unit():
    """Rows of up to 8192 tokens, bf16 and fp32: 1024 threads with at most 64 registers."""
    for name, k in of("evict_select").items():
        threads, quads, many, fp8 = map(int, re.search(r"evict_selectILi(\d+)ELi(\d+)ELb(\d)ELb(\d)E", name).groups())
        if threads == 1024 and quads <= 2 and not fp8:
            assert workgroups(k) >= 8 and k[".vgpr_spill_count"] == 0, (name, k[".vgpr_count"])
