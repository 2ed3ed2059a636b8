"""CPU-only: registers of the 4-bit cache's kernels, from the metadata in the library's own code objects."""
import re

from test_kernel_registers import kernels, spills  # noqa: F401


def test_cache_kernels_hold_their_registers(spills):  # noqa: F811
    """None spills but the kernel for many rows with fp16 results of 128 elements, whose queries are two fp16 numbers: 15 at most, as measured."""
    forms = {k: v for k, v in spills.items() if "k_kv4_" in k}
    assert len(forms) >= 80
    two = {k: v for k, v in forms.items() if re.search(r"k_kv4_promptILi128ELi[48]ELi1ELb1E", k)}
    assert len(two) == 4 and max(two.values()) <= 15, two
    assert {k: v for k, v in forms.items() if v and k not in two} == {}


def test_attention_kernels_leave_a_unit_two_workgroups(kernels):  # noqa: F811
    """Two waves a SIMD: eight tiles of codes of a compute unit are under way to memory."""
    forms = {k: v[0] for k, v in kernels.items() if "k_kv4_attention" in k}
    assert len(forms) >= 48 and max(forms.values()) <= 256
