"""Rows whose best column has nearly all the probability: the results keep to their signs (a log probability is never
above zero, an entropy and a log sum about the maximum never below) and to the bounds of the other tests."""
import math

import pytest
import torch

import token_reference as R
from paper_2608_00977_b200 import binding as B
from test_gpu_token_ops import DEV, _check_logprobs, _gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("rest", [1e-2, 1e-6, 1e-9, 0.0])
@pytest.mark.parametrize("scale", [1.0, 0.7, 3.0])
@pytest.mark.parametrize("n,v", [(40, 2003), (2000, 517), (4, 100_003)])
def test_confident_rows(dtype, rest, scale, n, v):
    g = _gen(n + v)
    x = torch.randn(n, v, generator=g, device=DEV) * 2
    y = torch.randint(0, v, (n,), generator=g, device=DEV)
    above = torch.logsumexp(x.double() * scale, dim=1) / scale - math.log(rest) / scale if rest else torch.full((n,), 1e4, device=DEV)
    x.scatter_(1, y[:, None], above.float()[:, None])
    x = x.to(dtype)
    r = _check_logprobs(x, y, 5, scale)
    assert (r.logprob <= 0).all() and (r.top_logprob <= 0).all()
    assert (r.entropy >= 0).all() and (r.log_sum >= 0).all()
    assert torch.equal(r.top_id[:, 0].long(), y) and torch.equal(r.top_logprob[:, 0], r.logprob)


@pytest.mark.parametrize("n,v", [(3, 1), (500, 1), (3, 9)])
def test_one_column_left(n, v):
    """A certain row: log probability and log sum are zero (the one term over itself).  The entropy is the rounding of one
    product 2^t t against its exact value, |t| <= 2^-5: at most 2^-29."""
    x = torch.full((n, v), -math.inf, device=DEV)
    x[:, v // 2] = torch.randn(n, device=DEV) * 1e3
    r = B.tsid_token_logprobs(x, torch.full((n,), v // 2, device=DEV), top_k=1, rank=True)
    for t in (r.logprob, r.log_sum, r.top_logprob):
        assert not t.any()
    assert (r.entropy >= 0).all() and (r.entropy <= 2.0 ** -29).all()
