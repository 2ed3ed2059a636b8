"""CPU-only: registers of the kernels over long contexts, from the metadata in the library's own code objects."""
from test_kernel_registers import kernels, spills  # noqa: F401


def test_prefix_kernel_for_many_rows_holds_most(spills):  # noqa: F811
    """Prefixes and many rows: partial results and the rows' own places take what the loop leaves; 22 registers at most, as measured, at 64 elements none."""
    forms = {k: v for k, v in spills.items() if "k_prefix_many" in k}
    assert len(forms) == 22 and max(forms.values()) <= 22, forms
    assert {k: v for k, v in forms.items() if v and "ILi128E" not in k} == {}


def test_workgroups_that_a_unit_holds(kernels):  # noqa: F811
    """Two waves a SIMD, of the weights' kernel for single queries three, of selection and eviction as many as there are rows for."""
    vgprs = {k: v[0] for k, v in kernels.items()}
    for name, forms, most in (("k_kv4_prefixI", 24, 256), ("k_kv4_prefix_separateI", 48, 256), ("k_kv4_weights_manyI", 4, 256), ("k_kv4_weightsI", 24, 170),
                              ("k_kv4_selectI", 6, 128), ("k_kv4_evict", 6, 96)):
        mine = {k: v for k, v in vgprs.items() if name in k}
        assert len(mine) == forms and max(mine.values()) <= most, (name, mine)
