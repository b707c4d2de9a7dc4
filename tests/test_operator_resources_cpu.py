"""What the kernels of the operators on tokens take of a compute unit, from the metadata of the library's code objects (no GPU)."""
from test_kernel_resources_cpu import kernels  # noqa: F401  (a fixture)


def test_no_value_of_the_operators_kernels_lives_in_memory(kernels):  # noqa: F811
    """But for fp32 walks with 96 rows of a state and two tiles of columns, which two workgroups on a unit repay."""
    names = ("walk_kernel<", "join_kernel", "sum_heads_kernel<", "step_kernel<", "lookup_kernel<", "few_tokens_kernel<", "sum_runs_kernel<", "join_runs_kernel<")
    found = {n: k for n, k in kernels.items() if n.startswith(names)}
    assert all(any(n.startswith(name) for n in found) for name in names)
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0 or (n.startswith("walk_kernel<3, 96, 2, true, true>") and k[".private_segment_fixed_size"] <= 128), n


def test_walks_up_to_128_rows_leave_room_for_two_workgroups(kernels):  # noqa: F811
    walks = {n: k for n, k in kernels.items() if n.startswith(("walk_kernel<1, ", "walk_kernel<4, ")) and int(n.split(",")[1]) <= 128}
    assert len(walks) >= 32
    for n, k in walks.items():
        assert k[".vgpr_count"] <= 256 and k[".group_segment_fixed_size"] <= 80 * 1024, n
