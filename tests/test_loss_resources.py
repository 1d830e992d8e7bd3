"""What the compiler made of the norm's and the class losses' kernels (no GPU needed): nothing may spill to scratch, and large tiles must leave room for two
workgroups on a CU: one fetches while the other multiplies."""
import pytest

from test_kernel_resources import resource_usage


@pytest.mark.parametrize("source,kernels", [("bgl_norm.hip", ("k_norm_forward", "k_norm_backward", "k_norm_reduce")),
                                            ("bgl_classes.hip", ("k_class_scores", "k_class_scores_stage", "k_class_top", "k_class_merge", "k_class_finish", "k_class_fix",
                                                                 "k_class_products", "k_class_products_stage", "k_class_reduce", "k_class_lay", "k_class_largest",
                                                                 "k_class_halves", "k_class_split", "k_class_zero"))])
def test_no_kernel_of_the_losses_spills(source, kernels):
    use = resource_usage(source)
    for name in kernels:
        assert any(f"{len(name)}{name}I" in k or f"{len(name)}{name}E" in k for k in use), name
    for name, u in use.items():
        assert u["ScratchSize"] == 0, (name, u)
        if "_stage" in name:
            assert u["Occupancy"] >= 2 and u["LDS Size"] <= 80 * 1024, (name, u)
        elif "k_class_scores" in name or "k_class_products" in name:
            assert u["Occupancy"] >= 2 and u["LDS Size"] <= 80 * 1024, (name, u)
