"""What the compiler made of the matrix kernels of a table as a model's layers: their speed hangs on two workgroups to a compute unit and on nothing of their
sums being kept in memory.  No GPU needed."""
from test_kernel_resources import kernels  # noqa: F401  (the fixture)

LDS = 160 * 1024          # of a compute unit


def _of(kernels, name):  # noqa: F811
    found = {n: k for n, k in kernels.items() if name in n}
    assert found
    return found


def test_matrix_kernels_keep_their_sums_in_registers(kernels):  # noqa: F811
    for name in ("k_logits", "k_product", "k_few", "k_embed_reduce", "k_adamw"):
        for n, k in _of(kernels, name).items():
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n


def test_two_workgroups_of_a_matrix_kernel_share_a_compute_unit(kernels):  # noqa: F811
    """One workgroup's exponentials run beside the other's products: 256 registers a lane and half of LDS each."""
    held, tiles, products = (_of(kernels, name) for name in ("13k_logits_held", "8k_logits", "9k_product"))
    assert (len(held), len(tiles), len(products)) == (10, 8, 12)
    for n, k in {**held, **tiles, **products}.items():
        if "k_logitsILi2ELi2ELi4ELi1ELi2E" in n:               # three parts, up to 64 tokens: one workgroup, a tile as large as LDS holds
            continue
        assert k[".vgpr_count"] <= 256 and k[".group_segment_fixed_size"] <= LDS // 2, n
