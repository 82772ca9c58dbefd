"""What the compiler makes of the attention kernel for tiles of 64 rows: nearly all registers of a wave are in use, and one that is spilled in
the loop would be read back behind the blocks in flight (twice the time, measured).  Compiles the file to assembly; needs no GPU."""
from test_kernel_code import _kernels


def test_nothing_passes_through_scratch_memory():
    kernels = _kernels("kv4_tile.hip")
    tiles = [name for name in kernels if "kv4_tile_kernel" in name]
    assert len(tiles) == 3
    for name in tiles:
        found = [i for i in kernels[name] if i.startswith(("flat_load", "flat_store", "scratch_load", "scratch_store"))]
        assert not found, (name, found)
