"""Registers of the kernels that normalise, answer and clip, read as in test_kernel_registers:
none of these keeps any in memory."""
import re

from test_kernel_registers import kernels, waves  # noqa: F401


def test_norms_answers_and_clipping_keep_nothing_in_memory(kernels):  # noqa: F811
    seen, lost = {}, []
    for name, (vgprs, scratch) in kernels.items():
        m = re.search(r"\bk_(rms|rms_backward|rms_reduce|to_bytes|from_bytes|lp_rows|lp_select|lp_merge"
                      r"|lp_top|squares|norm_factor|norm_small|scale)\b", name)
        if m is None:
            continue
        seen[m[1]] = seen.get(m[1], 0) + 1
        # workgroups of 1024 threads need four waves on each SIMD
        if scratch > 0 or (m[1] in ("lp_select", "norm_factor", "norm_small") and waves(vgprs) < 4):
            lost.append((name[:90], vgprs, scratch))
    assert len(seen) == 13 and not lost, (seen, lost)
