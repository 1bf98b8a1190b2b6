"""Registers of the softmax head's kernels, read as in test_kernel_registers: those
that stream records through LDS are made for a number of waves per SIMD (a template
argument), and keep no more than a few registers in memory."""
import re

from test_kernel_registers import kernels, waves  # noqa: F401


def test_softmax_kernels_keep_their_waves(kernels):  # noqa: F811
    seen, lost = 0, []
    for name, (vgprs, scratch) in kernels.items():
        m = re.search(r"k_sm_(lse|grad)<(unsigned short|float), (\d+), (\d+), (\d+), (\d+), true",
                      name)
        if m is None:
            continue
        seen += 1
        if waves(vgprs) < int(m[6]) or scratch > 16:
            lost.append((name[:90], vgprs, scratch))
    assert seen >= 30 and not lost, lost


def test_the_others_keep_nothing_in_memory(kernels):  # noqa: F811
    seen = 0
    for name, (_, scratch) in kernels.items():
        if re.search(r"k_(norm|norm_backward|adamw|adamw_state|sm_few|sm_pack|sm_join|sm_loss)<",
                     name):
            seen += 1
            assert scratch == 0, name[:90]
    assert seen >= 60
