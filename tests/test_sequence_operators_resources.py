"""What the compiler made of the kernels of a model of word sequences: nothing that they hold in registers goes to memory and back.  No GPU needed."""
from test_kernel_resources import kernels  # noqa: F401  (the fixture)


def _of(kernels, name):  # noqa: F811
    found = {n: k for n, k in kernels.items() if name in n}
    assert found
    return found


def test_registers_stay_registers(kernels):  # noqa: F811
    for name in ("6k_norm", "11k_norm_grad", "9k_dropout", "7k_recur", "12k_recur_grad", "12k_recur_step", "10k_draw_top", "11k_draw_bins", "13k_draw_border", "13k_draw_gather", "6k_draw"):
        for n, k in _of(kernels, name).items():
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n


def test_workgroups_of_the_recurrence_share_a_compute_unit(kernels):  # noqa: F811
    """One workgroup's loads run beside another's waiting: two of 512 threads (128 registers a thread) forward in bfloat16, four of 256 else, three for fp32 gradients."""
    for n, k in _of(kernels, "7k_recurI").items():
        assert k[".vgpr_count"] <= 128 and k[".group_segment_fixed_size"] <= 40 * 1024, n
    for n, k in _of(kernels, "12k_recur_gradI").items():
        assert k[".vgpr_count"] <= (128 if "gradIt" in n else 168) and k[".group_segment_fixed_size"] <= 40 * 1024, n
