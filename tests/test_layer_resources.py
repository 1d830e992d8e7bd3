"""What the compiler made of the layers' kernels (no GPU needed): nothing may spill to scratch, and the large tiles of the row
products must leave room for three workgroups on a CU: with two they took a quarter longer."""
import re

import pytest

from test_kernel_resources import resource_usage


@pytest.mark.parametrize("source,kernels", [("bgl_linear.hip", ("k_linear_rows", "k_linear_dw", "k_linear_dz", "k_linear_reduce", "k_group_place")),
                                            ("bgl_orthogonal.hip", ("k_ortho_norm", "k_ortho_start", "k_ortho_product", "k_ortho_whole"))])
def test_no_kernel_of_the_layers_spills(source, kernels):
    use = resource_usage(source)
    for name in kernels:
        assert any(name in k for k in use), name
    for name, u in use.items():
        assert u["ScratchSize"] == 0, (name, u)
        # forward products with 128 x 128 tiles (cut <2, 2, 4, 4>)
        if re.search(r"k_linear_rows.*Lb0E.*CutILi2ELi2ELi4ELi4E", name):
            assert u["Occupancy"] >= 3 and u["LDS Size"] <= 160 * 1024 // 3, (name, u)


def test_every_row_product_keeps_its_workgroups_on_a_cu():
    """Row products of one team: three workgroups of large tiles on a CU, two where dz is made on the way (rows of dy and of z wait in registers
    side by side), five of small tiles, four with dz; dW: two."""
    least, seen = {(128, "0"): 3, (128, "1"): 2, (64, "0"): 5, (64, "1"): 4}, set()
    for name, u in resource_usage("bgl_linear.hip").items():
        m = re.search(r"k_linear_rows.*CutILi(\d)ELi\dELi(\d)ELi\dEEELb\dELi1ELb(\d)E", name)
        if m:
            kind = 16 * int(m.group(1)) * int(m.group(2)), m.group(3)        # rows of a tile; dz or not
            seen.add(kind)
            assert u["Occupancy"] >= least[kind], (kind, name, u)
        if "k_linear_dw" in name:
            assert u["Occupancy"] >= 2, (name, u)
    assert seen == set(least)
