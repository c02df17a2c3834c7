"""The kernels of the 8-bit checkpoints and of the cross entropy: nothing in scratch memory."""
from test_kernel_resources import resources   # compiled once for both files


def test_they_use_no_scratch_memory():
    kinds = ("act8_pack_kernel", "act8_unpack_kernel", "gated_fwd_kernel", "gated_bwd_kernel", "add_parts_kernel", "ce_select_kernel",
             "ce_gather_kernel", "ce_piece_stats_kernel", "ce_piece_grad_kernel", "ce_finish_kernel", "ce_add_kernel", "ce_scatter_kernel")
    res = resources()
    for kind in kinds:
        found = {n: r for n, r in res.items() if kind in n}
        assert found, kind
        assert all(r.get("scratch", -1) == 0 and r.get("vgpr_spill", -1) == 0 for r in found.values()), found
