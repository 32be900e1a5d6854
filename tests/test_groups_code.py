"""What the linear layer with a step per group was compiled to, read from the library that was built here."""
from test_qgemm_code import _metadata, code_objects  # noqa: F401  (a fixture)


def test_no_register_is_spilled(code_objects):
    """A reload waits for every load in flight: for the weights and rows that were requested ahead."""
    kernels = list(_metadata(code_objects, "linear_groups_"))
    spilled = [n for n, m in kernels if m["vgpr_spill_count"] or m["private_segment_fixed_size"]]
    assert kernels and not spilled, spilled
