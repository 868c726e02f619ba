"""Scratch memory of the 4-bit cache's and sampled acceptance's kernels, from
the built library's metadata: none but what is named here."""
from test_kernel_resources_cpu import _kernels

# kernel -> bytes of scratch a thread at most, and what lies there
KNOWN = {
    "kvq_score_kernelILi1ELi3EE": 60,    # float32 queries' addresses and parts, between the passes over the blocks
    "sample_node_kernelILb1EE": 96,      # two of eight chunks' weights, read again in each sum over the row
}


def test_only_the_known_kernels_use_scratch():
    mine = [k for k in _kernels() if "kvq" in k[".name"] or "sample_" in k[".name"]]
    for part in ("kvq_score_kernel", "kvq_attention_kernel", "kvq_store_kernel", "kvq_gather_kernel", "kvq_select_kernel",
                 "sample_node_kernel", "sample_part_kernel", "sample_walk_kernel"):
        assert any(part in k[".name"] for k in mine), part
    for k in mine:
        most = max([n for part, n in KNOWN.items() if part in k[".name"]] + [0])
        assert k[".private_segment_fixed_size"] <= most, (k[".name"], k[".private_segment_fixed_size"])
    for part in KNOWN:  # none that is listed without need
        assert any(part in k[".name"] and k[".private_segment_fixed_size"] for k in mine), part
