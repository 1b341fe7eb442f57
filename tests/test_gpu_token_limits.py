"""Operators on factor rows and score rows: arguments that the Python layer refuses before the call."""
import pytest
import torch

from paper_2608_00977_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_matrices_beyond_the_interface_are_refused():
    """2^32 + 8 rows or columns were taken for 8.  (One matrix of 8.6 GB, of which nothing is read.)"""
    big = torch.empty(2 ** 32 + 8, dtype=torch.bfloat16, device=DEV)
    table, scores = big.view(-1, 1), big.view(1, -1)
    ids = torch.tensor([3, 20], device=DEV)
    one = torch.zeros(1, device=DEV)
    listed = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    for call in (lambda: B.tsid_embed(table, ids),
                 lambda: B.tsid_embed(scores, ids, out=torch.empty(2, 8, device=DEV)),
                 lambda: B.tsid_embed_grad(torch.zeros(2, 1, device=DEV), ids, 2 ** 32 + 8, out=table),
                 lambda: B.tsid_token_logprobs(scores),
                 lambda: B.tsid_token_logprobs_grad(scores, None, one, one, out=scores),
                 lambda: B.tsid_distill(scores, listed, one.view(1, 1))):
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_a_list_that_is_not_a_tensor_is_refused():
    x = torch.zeros(2, 5, device=DEV)
    for ids, lp in ((None, None), ([[0], [1]], x[:, :1].contiguous()), (torch.zeros(2, 1, dtype=torch.int32, device=DEV), None)):
        with pytest.raises(ValueError):
            B.tsid_distill(x, ids, lp)
