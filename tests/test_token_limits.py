"""Operators on factor rows and score rows without a GPU: sizes at the limits of the interface are refused before any
CUDA call, or reported as documented."""
import pytest

from paper_2608_00977_b200 import binding as B

P = 1 << 20      # an address that is never read: the calls below are refused first


@pytest.fixture(scope="module")
def L():
    import __graft_entry__ as g
    g.build()
    return B.lib()


@pytest.mark.parametrize("dim", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 31 - 512, 2 ** 31 - 1023])
def test_lookup_refuses_rows_whose_indices_would_leave_32_bits(L, dim):
    assert L.tsid_embed(4, 10, dim, P, 1, dim, P, 0, -1, 1.0, P, 1, dim, None, None) == B.TSID_ERR_UNSUPPORTED
    assert b"dim" in L.tsid_last_error(None)
    assert L.tsid_embed(0, 10, 2 ** 31 - 1024, None, 1, 0, None, 0, -1, 1.0, None, 1, 0, None, None) == B.TSID_OK


@pytest.mark.parametrize("rows,dim", [(2 ** 32 + 10, 8), (2 ** 31, 8), (10, 2 ** 32 + 8), (-2 ** 32 + 5, 8)])
def test_sizes_beyond_the_interface_are_not_cut_to_32_bits(L, rows, dim):
    """(2^32 + 10 rows were taken for 10.)"""
    with pytest.raises(ValueError, match="2\\^31"):
        B.tsid_embed_grad_workspace_bytes(1000, rows, dim)


def test_a_small_batch_needs_no_workspace_below_2_24_rows(L):
    """256 tokens fit one launch while a row number and a token's place fit one word."""
    for tokens, rows, none in ((256, 2 ** 24 - 1, True), (256, 2 ** 24, False), (257, 2 ** 24 - 1, False), (1, 2 ** 24, False),
                               (0, 10, True)):
        need = B.tsid_embed_grad_workspace_bytes(tokens, rows, 8)
        assert (need == 0) == none, (tokens, rows, need)
    assert L.tsid_embed_grad(256, 2 ** 24, 8, P, 0, 8, P, 0, -1, 1.0, P, 0, 8, 0, None, 0, None, None) == B.TSID_ERR_INVALID_ARG
    assert b"workspace" in L.tsid_last_error(None)
