"""Sizes at the edges of the cached operators' supported range: refusals and workspace sizes,
without a GPU."""
import pytest

from paper_2609_08443_amd import sa_sketch as sa

P = 1 << 12
SIZES = {"fwd": sa.stca_cached_fwd_workspace_size, "bwd": sa.stca_cached_bwd_workspace_size}


@pytest.mark.parametrize("way", ["fwd", "bwd"])
def test_rows_of_the_softmax_at_the_edge_of_a_launch(way):
    """Separate products give four rows a workgroup of 256 threads; 2^24 workgroups are 2^32 threads,
    more than a launch holds, from 2^26 - 3 rows on."""
    size = SIZES[way]
    assert 8191 * 8193 == 2 ** 26 - 1 and 16380 * 4097 == 2 ** 26 - 4
    assert size(8191, 8193, 1, 8, 1, 1) == 0
    assert size(16380, 4097, 1, 8, 1, 1) > 0
    L = sa.lib()
    head = [P, P, 4, P, 0, P, P, P, P, 8191, 8193, 1, 8, 1, 1.0, 1]
    rc = L.sa_stca_cached_fwd(*head, P, 1, None, P, 1 << 60, None) if way == "fwd" else \
        L.sa_stca_cached_bwd(*head, P, P, P, P, P, 1, P, 1 << 60, None)
    assert rc == 2 and L.sa_last_error().decode() != ""


def test_padded_targets_within_their_index():
    """The last targets' copies, 64 rows of h D, h D and four times D values, are counted in 16-byte
    pieces in 32 bits; where they are more (heads of 8 at D = 32768: 2^31 + 2^20) none are made, and
    a 65th target takes no more workspace than its own rows."""
    def last(D, h):
        return SIZES["bwd"](1, 65, 4, D, h, sa.SA_BF16) - SIZES["bwd"](1, 64, 4, D, h, sa.SA_BF16)

    def copies(D, h):
        return 64 * 2 * (2 * h + 4) * D

    def own(D, h):   # C, dU, U, dC; q W_Q, dQp, q, dout; rows of four keys
        return 2 * (4 * h + 4) * D + (4 + 4 * 12) * h + 16 * 256
    assert copies(32768, 4096) // 16 >= 2 ** 31
    assert 0 < last(32768, 4096) <= own(32768, 4096)
    assert copies(32768, 2048) // 16 < 2 ** 31
    assert copies(32768, 2048) <= last(32768, 2048) <= copies(32768, 2048) + own(32768, 2048)
