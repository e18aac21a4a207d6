"""What the kernels of prompt attention, tree attention and moves need, where their launch rules count on it."""
from test_kernel_resources import kernels  # noqa: F401


def per_simd(kernels, name, waves):
    """Wavefronts of a kernel that a SIMD holds: 512 registers a lane in steps of eight, 160 KiB of LDS a compute unit."""
    k = kernels[name]
    groups = 160 * 1024 // max(1, k["group_segment_fixed_size"])
    return min(512 // ((k["vgpr_count"] + 7) // 8 * 8), groups * waves // 4)


def test_prompt(kernels):
    """`slots`: two workgroups of 128 rows a compute unit, one of fewer rows."""
    assert per_simd(kernels, "kvq_prompt_kernel<2, 4, 1, 2>", 4) == 2
    for shape in ("1, 1, 4, 4", "2, 1, 4, 4", "2, 2, 2, 4"):
        assert per_simd(kernels, f"kvq_prompt_kernel<{shape}>", 4) == 1


def test_tree(kernels):
    """Twelve wavefronts a compute unit, in three workgroups or one; two workgroups of few rows."""
    for scales in (4, 2):
        assert per_simd(kernels, f"kvq_tree_shared_kernel<2, false, {scales}, 1, 4>", 4) == 3
        assert per_simd(kernels, f"kvq_tree_shared_kernel<2, false, {scales}, 1, 12>", 12) == 3
        assert per_simd(kernels, f"kvq_tree_shared_kernel<2, true, {scales}, 1, 4>", 4) == 2
    assert per_simd(kernels, "kvq_tree_shared_kernel<2, false, 4, 2, 4>", 4) == 3
    assert per_simd(kernels, "kvq_tree_shared_kernel<2, true, 4, 2, 4>", 4) == 2
    for rows in (1, 2):
        assert per_simd(kernels, f"kvq_tree_kernel<{rows}, false>", 4) == 2
        assert per_simd(kernels, f"kvq_tree_kernel<{rows}, true>", 4) == 1


def test_no_kernel_that_no_launch_reaches(kernels):
    made = {n for n in kernels if n.startswith(("kvq_prompt", "kvq_tree", "kvq_fork", "kvq_read", "kvq_clear"))}
    shared = {f"kvq_tree_shared_kernel<2, {i16}, {scales}, 1, 4>" for i16 in ("true", "false") for scales in (4, 2)}
    assert made == shared | {f"kvq_tree_shared_kernel<2, {i16}, 4, 2, 4>" for i16 in ("true", "false")} | {
        f"kvq_tree_shared_kernel<2, false, {scales}, 1, 12>" for scales in (4, 2)} | {
        f"kvq_tree_kernel<{rows}, {i16}>" for rows in (1, 2) for i16 in ("true", "false")} | {"kvq_tree_merge_kernel"} | {
        f"kvq_prompt_kernel<{shape}>" for shape in ("1, 1, 4, 4", "2, 1, 4, 4", "2, 2, 2, 4", "2, 4, 1, 2")} | {
        f"kvq_prompt_merge_kernel<{rows}>" for rows in (16, 32, 64, 128)} | {
        "kvq_fork_kernel<true>", "kvq_fork_kernel<false>", "kvq_fork_table_kernel", "kvq_read_kernel", "kvq_clear_tail_kernel"}
