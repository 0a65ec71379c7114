"""What the compiler reports for the kernels of the batch calls, against the workgroups per compute unit that their planner counts on."""
from tests.test_kernel_resources_cpu import LDS, OCC, SCRATCH, _args, table  # noqa: F401 (a fixture)


def rows_of(table, kernel):  # noqa: F811
    rows = {n: r for n, r in table.items() if kernel in n}
    assert rows, kernel
    return rows


def test_few_rows_kernel_two_workgroups_per_compute_unit(table):  # noqa: F811
    """Workgroups of four waves: two fit by registers (two waves per SIMD) and by LDS, at every head dimension and rank."""
    rows = rows_of(table, "batch_rows_kernel")
    assert len(rows) == 24
    for name, row in rows.items():
        assert row[SCRATCH] == 0 and row[OCC] >= 2 and row[LDS] <= 80 * 1024, (name, row)


def test_tile_walking_kernel_two_workgroups_per_compute_unit(table):  # noqa: F811
    """... but one of the rotated key side at d = 128 and ranks above 32, which the plan counts so."""
    rows = rows_of(table, "batch_tiles_kernel")
    one = 0
    for name, row in rows.items():
        d, rp, _, _, _, _, rope = _args(name)
        two = not (rope and d == 128 and rp == 64)
        one += not two
        assert row[SCRATCH] == 0 and row[OCC] >= (2 if two else 1) and row[LDS] <= (80 if two else 160) * 1024, (name, row)
    assert one == 3


def test_key_weights_kernels(table):  # noqa: F811
    """Statistics: three workgroups of four waves per compute unit, two at d = 128 and ranks above 32; sums: two."""
    for name, row in rows_of(table, "weights_stats_mfma_kernel").items():
        d, rp = _args(name)[:2]
        per_unit = 2 if (d, rp) == (128, 64) else 3
        assert row[SCRATCH] == 0 and row[OCC] >= per_unit and row[LDS] * per_unit <= 160 * 1024, (name, row)
    for kernel in ("weights_sum_mfma_kernel", "weights_sum_rows_kernel"):
        for name, row in rows_of(table, kernel).items():
            assert row[SCRATCH] == 0 and row[OCC] >= 2 and row[LDS] <= 80 * 1024, (name, row)
