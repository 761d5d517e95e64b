"""What the compiler gave the kernels of RMSNorm, the cross-entropy of a linear layer and the clipping: no GPU needed."""
import re

from test_kernel_resources import kernels      # noqa: F401


def test_no_kernel_needs_scratch(kernels):      # noqa: F811
    """(none has an array that is indexed at run time, so scratch would be registers that do not fit)"""
    own = {n: v for n, v in kernels.items() if re.search(r"\d(ce|small|few|rms|clip)_[a-z0-9_]*kernel", n)}
    names = {re.search(r"\d((?:ce|small|few|rms|clip)_[a-z0-9_]*kernel)", n).group(1) for n in own}
    assert {"ce_logits_kernel", "ce_grads_kernel", "ce_pack_kernel", "ce_colmax_kernel", "ce_transpose_kernel", "ce_turn_kernel", "ce_join_kernel", "ce_sums_kernel", "small_logits_kernel",
            "small_rows_kernel", "small_turn_kernel", "few_grads_kernel", "few_sums_kernel", "rms_fwd_kernel", "rms_bwd_kernel", "clip_norm_kernel", "clip_scale_kernel"} <= names
    assert {n: v for n, v in own.items() if v != (0, 0)} == {}
