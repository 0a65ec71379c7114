"""What the compiler reports for the kernels of the 8-bit calls, against the workgroups per compute unit that their planner counts on."""
from tests.test_batch_resources_cpu import rows_of
from tests.test_kernel_resources_cpu import LDS, OCC, SCRATCH, _args, table  # noqa: F401 (a fixture)


def test_few_rows_kernels_two_workgroups_per_compute_unit(table):  # noqa: F811
    """... but one of 32 rows to a wave at ranks above 32."""
    rows = rows_of(table, "attn8_rows_kernel")
    assert len(rows) == 24
    for name, row in rows.items():
        assert row[SCRATCH] == 0 and row[OCC] >= 2 and row[LDS] <= 80 * 1024, (name, row)
    rows = rows_of(table, "attn8_rows32_kernel")
    assert len(rows) == 48
    for name, row in rows.items():
        d, _, rp = _args(name)[:3]
        per_unit = 1 if rp == 64 else 2
        assert row[SCRATCH] == 0 and row[OCC] >= per_unit and row[LDS] * per_unit <= 160 * 1024, (name, row)


def test_tile_walking_kernels_two_workgroups_per_compute_unit(table):  # noqa: F811
    for name, row in rows_of(table, "attn8_tiles_kernel").items():
        assert row[SCRATCH] == 0 and row[OCC] >= 2 and row[LDS] <= 80 * 1024, (name, row)


def test_products_of_integers(table):  # noqa: F811
    """A workgroup of eight waves per compute unit with its stages in LDS, two of the kernel for few tokens and of tiles of 32."""
    for kernel in ("matmul_i8_small_kernel", "matmul_i8_chain_kernel", "matmul_i8_wide_kernel"):
        for name, row in rows_of(table, kernel).items():
            assert row[SCRATCH] == 0 and row[OCC] >= 2 and row[LDS] <= 128 * 1024, (name, row)
    assert sum(row[OCC] >= 4 and row[LDS] <= 80 * 1024 for row in rows_of(table, "matmul_i8_small_kernel").values()) == 2
    for name, row in rows_of(table, "matmul_i8_stream_kernel").items():
        assert row[SCRATCH] == 0 and row[OCC] >= 2 and row[LDS] <= 80 * 1024, (name, row)


def test_appending_and_reading_back(table):  # noqa: F811
    for kernel in ("cache8_append_kernel", "cache8_gather_kernel", "quantize_rows_kernel", "attn8_vector_kernel"):
        for name, row in rows_of(table, kernel).items():
            assert row[SCRATCH] == 0 and row[OCC] >= 3, (name, row)
