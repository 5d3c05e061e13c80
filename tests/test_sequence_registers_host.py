"""CPU test: vector registers of the sequence layers' kernels (test_kernel_registers_host.py says why and how)."""
import re

import pytest

from test_kernel_registers_host import kernels  # noqa: F401  (a fixture)

# (mangled name, how many instantiations, most registers)
FIT = [
    (r"_Z19product_rows_kernelILi[2345]ELb[01]EE.*", 8, 128),              # four waves a SIMD
    (r"_Z30inner_product_pair_(rows|wide)_kernelILi[2345]ELi[56]EE.*", 16, 128),
    (r"_Z25final_inverse_(rows|wide)_kernelILi[2345]EE.*", 8, 96),         # five
    (r"_Z18centre_rows_kernelILi[2345]ELb[01]EE.*", 8, 72),                # seven
    (r"_Z31inner_product_sum_halves_kernelILi[123]ELb[01]EE.*", 6, 256),   # two workgroups of four waves
    (r"_Z17pair_inner_kernel.*", 1, 64),                                   # eight
    (r"_Z(20group_moments|17norm_times)_kernel.*", 2, 64),
]


@pytest.mark.parametrize("name,count,most", FIT)
def test_registers(kernels, name, count, most):  # noqa: F811
    which = {k: v for k, v in kernels.items() if re.fullmatch(name, k)}
    assert len(which) == count, sorted(which)
    for k, (used, spilled) in which.items():
        assert used <= most and spilled == 0, (k, used, spilled)
