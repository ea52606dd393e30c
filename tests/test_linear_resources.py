"""No kernel of the projections keeps registers in scratch memory."""
from paper_2110_09195_amd import binding
from test_kernel_resources import kernels


def test_projections_have_no_scratch():
    binding.lib()
    names = ("linear_", "low_few", "low_tile", "adapters_", "checkpoint_")
    ours = {n: k for n, k in kernels(binding.LIB_PATH).items() if any(part in n for part in names)}
    assert len(ours) >= 60, sorted(ours)
    spilled = {n: (k[".vgpr_spill_count"], k[".sgpr_spill_count"], k[".private_segment_fixed_size"]) for n, k in ours.items()
               if k[".vgpr_spill_count"] or k[".sgpr_spill_count"] or k[".private_segment_fixed_size"]}
    assert not spilled, spilled
