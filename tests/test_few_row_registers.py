"""Registers of the kernels for few rows: how many workgroups share a compute unit rests on them."""
import re

from test_kernel_registers import kernels, objects  # noqa: F401  (fixtures)

# kernel, element (f float, t bfloat16), groups of rows -> spilled vector registers; three of bfloat16 rows in two parts are written and read once for
# 32 rows, outside the loop over the steps
SPILLED = {("few_second", "t", 2): 3}


def test_two_workgroups_of_up_to_two_groups_fit_a_compute_unit(kernels):  # noqa: F811
    seen = {}
    for name, k in kernels.items():
        m = re.search(r"(few_first|few_second|few_linear)_kernelI(f|t)Li(\d)E", name)
        if m:
            key = (m[1], m[2], int(m[3]))
            seen[key] = seen.get(key, 0) + 1
            assert k[".vgpr_count"] <= (128 if key[2] <= 2 else 256), name
            assert k[".vgpr_spill_count"] <= SPILLED.get(key, 0), name
    assert all(seen.get((f, e, g)) for f in ("few_first", "few_second") for e in "ft" for g in (1, 2, 4))
    assert all(seen.get(("few_linear", e, g)) for e in "ft" for g in (1, 2))


def test_nothing_else_of_these_operators_is_spilled(kernels):  # noqa: F811
    found = 0
    for name, k in kernels.items():
        if re.search(r"few_(gate|route|join)_kernel|linear_finish|act_bwd|join_(columns|parts)|grad_(table|norm|join|scale)", name):
            found += 1
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
    assert found > 20
