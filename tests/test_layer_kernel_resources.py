"""What the compiler made of the norms', the dense layer's and the update's kernels (no GPU needed)."""
import pytest

from test_kernel_resources import kernels


@pytest.mark.parametrize("part,least", [("norm_fwd_kernel", 20), ("norm_bwd_kernel", 20), ("norm_bwd_pair_kernel", 20), ("norm_fwd_wide", 2), ("norm_bwd_rows", 2),
                                        ("norm_bwd_columns", 2), ("sum_partials", 1), ("dense_any", 4), ("dense_bwd_h", 1), ("dense_gemm256", 12), ("DenseWay", 40),
                                        ("adamw_runs", 1), ("adamw_matrices", 3), ("grad_squares", 1), ("grad_norm", 1)])
def test_no_scratch(part, least):
    found = {n: k for n, k in kernels().items() if part in n}
    assert len(found) >= least, (part, len(found))
    spilled = {n: k[".private_segment_fixed_size"] for n, k in found.items() if k[".private_segment_fixed_size"]}
    assert not spilled, spilled
