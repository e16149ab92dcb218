"""What the kernels for rows in 8 bits take of a compute unit."""
from test_kernel_resources import _registers, kernels  # noqa: F401  (kernels is a fixture)


def test_no_scratch_memory(kernels):  # noqa: F811
    """Registers and LDS hold everything; the largest gated form keeps six registers per lane in memory, none of them inside its loop."""
    mine = {n: k for n, k in kernels.items() if "rows8_" in n}
    of = lambda name: sum(name in n for n in mine)   # noqa: E731
    assert [of(n) for n in ("few", "waves", "tile", "rms", "store", "load")] == [4, 9, 14, 19, 3, 3]
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] <= (24 if "tile_kernel" in n and "Lb1ELi4ELi4E" in n else 0), n


def test_two_workgroups_of_tiles(kernels):  # noqa: F811
    """Tiles of 128 x 128 and 128 x 64 with two or three blocks on their way: two workgroups share a compute unit."""
    mine = {n: k for n, k in kernels.items() if "rows8_tile_kernel" in n and ("ELi2ELi2ELi2E" in n or "ELi2ELi1ELi3E" in n)}
    assert len(mine) == 6
    for n, k in mine.items():
        assert _registers(k) <= 256, (n, _registers(k))
