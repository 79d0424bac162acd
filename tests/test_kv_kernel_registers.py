"""Registers of the 4-bit cache's kernels that did not fit, as the compiler reports them.

The few rows' kernel with heads of 256 kept four groups' metadata, weights and codes at once and spilled 102 registers: 151 us
where a column for each row and group, without a spill, takes 91.
"""
from test_kernel_registers import kernels  # noqa: F401  (the fixture)


def test_kv_registers(kernels):  # noqa: F811
    kv = {n: v for n, v in kernels.items() if n.startswith("k_kv_")}
    assert {n.split("<")[0] for n in kv} == {"k_kv_append", "k_kv_read", "k_kv_plan", "k_kv_attend_few", "k_kv_attend_many", "k_kv_join"}
    for name, v in kv.items():
        if name.startswith("k_kv_attend_many"):  # addresses of the slow path, outside the rounds of two tiles
            assert v["vgpr_spill_count"] <= 24 and v["private_segment_fixed_size"] <= 100, (name, v)
        else:
            assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0, (name, v)
