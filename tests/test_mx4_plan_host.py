"""How a product with many vectors is cut, by the size of its workspace: the fragments of a
chunk of 64 columns and a tile of 32 vectors take 4096 bytes a piece."""
import pytest


@pytest.fixture(scope="module")
def sq():
    import os
    import paper_2609_38477_amd as sq
    if not os.path.exists(sq.LIB_PATH):
        from paper_2609_38477_amd import build
        build.build()
    return sq


@pytest.mark.parametrize("xtype,pieces,widths", [(0, 3, (2, 3)), (1, 2, (3, 4)), (2, 1, (3, 4))])
def test_counts_of_tiles_without_a_divisor_take_wide_ones(sq, xtype, pieces, widths):
    # a tall matrix is cut along its rows alone, so the workspace is the fragments
    for tiles in (5, 7, 11, 13, 17, 19, 23, 29, 31):
        nbytes = sq.seedq_mx4_gemv_workspace_bytes(128000, 4096, 32 * tiles, xtype)
        padded, rest = divmod(nbytes, 4096 * pieces * 64)
        assert rest == 0 and padded in {-(-tiles // w) * w for w in widths}, (tiles, padded)
        if pieces < 3:
            assert padded > tiles      # a tile of one would have none to spare


def test_workspaces_grow_with_what_they_hold(sq):
    for rows, cols in ((1001, 2056), (4096, 4096), (32000, 4096), (8192, 28672)):
        for xtype, pieces in ((0, 3), (1, 2), (2, 1)):
            for nvec in range(33, 600, 37):
                chunks = -(-cols // 128) * 2
                least = -(-nvec // 32) * 4096 * pieces * chunks
                got = sq.seedq_mx4_gemv_workspace_bytes(rows, cols, nvec, xtype)
                assert got % 256 == 0 and got >= least
