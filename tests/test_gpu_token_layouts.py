"""What layout may change: the same call gives the same bits; the same values in another layout may be added in another
order, within the bounds of any order."""
import pytest
import torch

import token_reference as R
from paper_2608_00977_b200 import binding as B
from test_gpu_token_ops import DEV, _gen, _ids, _within

pytestmark = pytest.mark.gpu


def _at(x, offset):
    """x in new memory, `offset` elements behind a 256-byte boundary."""
    buf = torch.empty(x.numel() + offset + 8, dtype=x.dtype, device=DEV)
    v = buf[offset:offset + x.numel()].view(x.shape)
    v.copy_(x)
    return v


@pytest.mark.parametrize("kind,tokens,rows,dim", [("one", 6000, 3, 64), ("skewed", 9000, 40, 64), ("skewed", 70_000, 300, 24)])
def test_gradient_of_the_lookup_in_other_layouts(kind, tokens, rows, dim):
    """fp32 rows of 64: 16-byte accesses at offset 0, 8-byte ones at offset 2 (other lanes per row, other borders), single
    elements at offset 1."""
    g = _gen(tokens)
    dy = torch.randn(tokens, dim, generator=g, device=DEV)
    ids = _ids(kind, tokens, rows, g)
    ref, bound = R.embed_grad(dy, ids, rows, 1.0)
    for a in (0, 2, 1):
        for b in (0, 2, 1):
            first = None
            for _ in range(2):
                out = _at(torch.full((rows, dim), float("nan"), device=DEV), b)
                B.tsid_embed_grad(_at(dy, a), ids, rows, out=out)
                _within(out, ref, bound + R.stored(ref, torch.float32), "gradient at %d, %d" % (a, b))
                assert first is None or torch.equal(out, first)
                first = out.clone()


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("n,v", [(3, 5003), (500, 1203), (2, 100_003)])
def test_statistics_of_rows_in_other_layouts(dtype, n, v):
    g = _gen(v)
    x = (torch.randn(n, v, generator=g, device=DEV) * 3).to(dtype)
    y = torch.randint(0, v, (n,), generator=g, device=DEV)
    ref = R.logprobs(x, y, 10, 1.0)
    bd = R.logprob_bounds(ref, v)
    for offset in range(8):
        r, again = (B.tsid_token_logprobs(_at(x, offset), y, top_k=10, rank=True) for _ in range(2))
        assert all(torch.equal(p, q) for p, q in zip(r, again))
        assert torch.equal(r.rank.long(), ref["rank"]) and torch.equal(r.top_id.long(), ref["top_id"])
        _within(r.log_sum, ref["log_sum"], bd["log_sum"], "log_sum")
        _within(r.entropy, ref["entropy"], bd["entropy"], "entropy")
