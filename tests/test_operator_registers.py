"""Registers of the int8 layers' and the sampler's kernels, instance by instance.  test_i8_host.py allows every instance what the largest needs;
what an instance that holds all its values today would begin to fetch back, only its own limit shows."""
import re

import pytest

from test_kernel_registers import kernels

SPILLED = {("i8_split_kernel", ""): 0, ("i8_whole_kernel", "jLi1"): 0, ("i8_whole_kernel", "jLi2"): 0, ("i8_whole_kernel", "mLi1"): 0,
           ("i8_whole_kernel", "mLi2"): 4,
           ("sample_kernel", "Lj256ELi8"): 0, ("sample_kernel", "Lj256ELi16"): 0, ("sample_kernel", "Lj256ELi32"): 0,
           ("sample_kernel", "Lj512ELi8"): 0, ("sample_kernel", "Lj512ELi16"): 0, ("sample_kernel", "Lj512ELi32"): 11,
           ("sample_kernel", "Lj1024ELi8"): 0, ("sample_kernel", "Lj1024ELi16"): 0, ("sample_kernel", "Lj1024ELi32"): 56}


@pytest.fixture(scope="module")
def built():
    return kernels()


@pytest.mark.parametrize("kernel,instance", SPILLED)
def test_no_instance_spills_more_than_it_did(built, kernel, instance):
    found = [k for name, k in built.items() if re.search(rf"\d+{kernel}I{instance}", name)]
    assert found
    for k in found:
        assert k[".vgpr_spill_count"] <= SPILLED[kernel, instance], (k[".name"], k[".vgpr_spill_count"])


def test_every_instance_has_a_limit(built):
    names = [n for n in built if re.search(r"\d+(i8_\w+_kernel|sample_kernel)I", n)]
    assert len(names) == 21                                         # 4 + 8 of the layers, 9 of the sampler
    assert all(sum(bool(re.search(rf"\d+{k}I{i}", n)) for k, i in SPILLED) == 1 for n in names)
