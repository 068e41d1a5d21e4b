"""Registers that the block operators' kernels spill (CPU: from libocc.so's own metadata): none, but where a comment of
csrc/norm.hip says so."""
import re

from test_kernel_registers_cpu import built, code_objects, kernels  # noqa: F401
from paper_2606_09200_amd import binding

# norm_gate_bwd_kernel<chunks, ragged end, activations, residual, direct>: t is bf16, f binary32
SPILLS = {("2", "t", "t", "1"): 16, ("2", "t", "f", "1"): 16, ("2", "t", "f", "0"): 1, ("1", "f", "f", "1"): 5}


def test_spilled_vector_registers(built):  # noqa: F811
    found = [k for elf in code_objects(binding.LIB_PATH) for k in kernels(elf)]
    ours = [k for k in found if any(n in k[".name"] for n in ("moe_", "norm_gate", "mx4_"))]
    assert len(ours) > 50
    for k in ours:
        m = re.search(r"norm_gate_bwd_kernelILi(\d)ELb(\d)E([tf])([tf])Lb(\d)E", k[".name"])
        allowed = SPILLS.get((m[1], m[3], m[4], m[5]), 0) if m else 0
        assert k.get(".vgpr_spill_count", 0) <= allowed, (k[".name"], k[".vgpr_spill_count"])
    assert sum("norm_gate_bwd_kernel" in k[".name"] for k in ours) == 24
