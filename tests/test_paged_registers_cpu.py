"""Registers that the paged cache's kernels spill (CPU: from libocc.so's own metadata): none to memory, but where a comment of
csrc/attn.hip says so."""
from test_kernel_registers_cpu import built, code_objects, kernels  # noqa: F401
from paper_2606_09200_amd import binding

SPILLS = {"attn_few_kernelILi256E": 1}


def test_spilled_vector_registers(built):  # noqa: F811
    found = [k for elf in code_objects(binding.LIB_PATH) for k in kernels(elf)]
    ours = [k for k in found if any(n in k[".name"] for n in ("kv_tables", "rope_kernel", "attn_few", "attn_pairs"))]
    assert len(ours) == 2 + 7 + 3 + 7
    for k in ours:
        allowed = sum(n for name, n in SPILLS.items() if name in k[".name"])
        assert k.get(".vgpr_spill_count", 0) <= allowed, (k[".name"], k[".vgpr_spill_count"])
        assert k[".private_segment_fixed_size"] <= 8 * allowed, k[".name"]
