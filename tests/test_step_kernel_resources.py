"""The kernels of attention, the vocabulary's table and the gradients' norm: nothing in scratch memory."""
from test_kernel_resources import resources   # compiled once for all files of its kind


def test_they_use_no_scratch_memory():
    kinds = ("attn_fwd_kernel", "attn_join_kernel", "attn_dq_kernel", "attn_dkv_kernel", "attn_parts_kernel", "embed_fwd_kernel", "embed_group_kernel",
             "embed_bwd_kernel", "embed_parts_kernel", "grad_squares_kernel", "grad_scale_kernel", "gram_kernel", "gram_sum_kernel", "grad_norm_kernel")
    res = resources()
    for kind in kinds:
        found = {n: r for n, r in res.items() if kind in n}
        assert found, kind
        assert all(r.get("scratch", -1) == 0 and r.get("vgpr_spill", -1) == 0 for r in found.values()), found
