"""What the kernels of the paged cache of 8-bit floating point need, where their launch rules count on it."""
from test_kernel_resources import kernels  # noqa: F401
from test_operator_resources import per_simd


def test_wavefronts(kernels):
    """Pieces of few rows: two workgroups a compute unit with blocks of 16 rows, one of 32; chunks: one, two wavefronts a SIMD; appends: five a SIMD."""
    assert per_simd(kernels, "kvq_paged8_ranges_kernel<1>", 8) == 4
    assert per_simd(kernels, "kvq_paged8_ranges_kernel<2>", 8) == 2
    for maps in (1, 2):
        assert per_simd(kernels, f"kvq_paged8_chunk_kernel<{maps}>", 8) == 2
    for tiles in (1, 2, 4, 8):
        assert 512 // ((kernels[f"kvq_paged8_append_kernel<{tiles}>"]["vgpr_count"] + 7) // 8 * 8) >= 5


def test_no_kernel_that_no_launch_reaches(kernels):
    assert {n for n in kernels if n.startswith("kvq_paged8")} == {f"kvq_paged8_{k}<{x}>" for k, xs in (
        ("ranges_kernel", "12"), ("chunk_kernel", "12"), ("append_kernel", "1248")) for x in xs} | {
        f"kvq_paged8_read_kernel<{wide}, {tiles}>" for wide in ("true", "false") for tiles in (1, 2, 4, 8)}
