"""No kernel of a network's ends keeps vector registers in scratch memory."""
from paper_2110_09195_amd import binding
from test_kernel_resources import kernels


def test_ends_of_a_network_have_no_scratch():
    binding.lib()
    ours = {n: k for n, k in kernels(binding.LIB_PATH).items() if any(part in n for part in ("vocab_tiles", "vocab_gradients", "embedding_", "loss_"))}
    assert len(ours) >= 46, sorted(ours)
    spilled = {n: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) for n, k in ours.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}
    assert not spilled, spilled
