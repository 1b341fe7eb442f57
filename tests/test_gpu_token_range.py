"""Operators on score rows over the whole accepted range of scores and scales: finite scores of any size give finite
statistics, as one finite mask value per column does (-1e10, -1e30), and so does any accepted scale."""
import math

import pytest
import torch

import token_reference as R
from paper_2608_00977_b200 import binding as B
from test_gpu_token_ops import DEV, _check_logprobs, _gen, _teacher
from test_gpu_token_ops import _within as _within_below_the_largest

pytestmark = pytest.mark.gpu

LEVELS = [-1e8, -1e10, 1e10, -1e12, -1e18, -1e20, -1e30, 1e30, -1e36]
PLACES = ["whole row", "first columns", "last columns", "every third run", "half of them"]


def _rows(place, level, n, v, dtype, g):
    """Ordinary scores with some columns at `level`.  The runs are long enough that a thread reads whole 16-byte
    chunks, and whole pairs of them, that hold nothing else."""
    x = torch.randn(n, v, generator=g, device=DEV) * 2
    col = torch.arange(v, device=DEV)
    at = {"whole row": col >= 0, "first columns": col < v // 2, "last columns": col >= v // 2,
          "every third run": col // 8 % 3 == 0}.get(place)
    if at is None:
        at = torch.rand(n, v, generator=g, device=DEV) < 0.5
    return torch.where(at, torch.full_like(x, level), x).to(dtype)


def _within(got, ref, bound, what):
    """As the other tests compare, except that a value beyond the type's largest is stored as infinite only from
    half a unit beyond it: below that the nearest value is the largest itself."""
    top = torch.finfo(got.dtype).max
    over = ref.abs() - top
    if got.dtype == torch.float16:      # 65504, whose unit is 32
        near = (over > 0) & (over < 16.0)
        ref = torch.where(near, ref.sign() * top, ref)
    _within_below_the_largest(got, ref, bound, what)


def _distill(x, ids, tlp, tail, scale, weight):
    """(loss, gradient, bound of the loss, bound of the gradient before storing) in 64 bits.  The mass outside the list
    is kept as a logarithm, because it can be far below the range of a 64-bit float; otherwise the terms and
    bounds are those of token_reference.distill."""
    n, v = x.shape
    ids, xd = ids.long(), x.double()
    valid = ids >= 0
    z = (xd - xd.max(dim=1, keepdim=True).values) * scale
    log_sum = z.exp().sum(dim=1, keepdim=True).log()
    lq = z - log_sum
    q = lq.exp()
    l = torch.where(valid, tlp.double(), -math.inf)
    if not tail:
        total = torch.logsumexp(l, dim=1, keepdim=True)
        l = torch.where(total > -math.inf, l - total, l)
    p = l.exp()
    pf = torch.zeros(n, v + 1, dtype=torch.float64, device=DEV).scatter_add_(1, torch.where(valid, ids, v), p)[:, :v]
    inside = torch.zeros(n, v + 1, dtype=torch.bool, device=DEV).scatter_(1, torch.where(valid, ids, v), True)[:, :v]
    out_max = xd.masked_fill(inside, -math.inf).max(dim=1, keepdim=True).values      # (every row has columns outside)
    zo = ((xd - out_max) * scale).masked_fill(inside, -math.inf)
    so = zo.exp().sum(dim=1, keepdim=True)
    share = zo.exp() / so                                                            # softmax outside the list
    lq_t = ((out_max - xd.max(dim=1, keepdim=True).values) * scale + so.log() - log_sum)[:, 0]
    p_t = (1.0 - p.sum(dim=1)).clamp(min=0.0) * tail
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    lqk = lq.gather(1, ids.clamp(0, v - 1))
    lt = torch.where(p_t > 0, (p_t.log() - lq_t).abs(), zero)
    loss = torch.where(p > 0, p * (l - lqk), zero).sum(dim=1) + torch.where(p_t > 0, p_t * (p_t.log() - lq_t), zero)
    grad = q * (p.sum(dim=1) + p_t)[:, None] - pf - p_t[:, None] * share
    fin, one = log_sum[:, 0].abs(), (ids.shape[1] + 16) * R.U32
    lk = torch.where(torch.isfinite(l), l.abs(), zero)
    b_loss = (p * (R.sum_bound(v) + one + 16 * R.U32 * (lqk.abs() + lk + fin[:, None]))).sum(dim=1) \
        + p_t * (R.sum_bound(v) + 8 * R.U32 * lq_t.abs()) + one * (lt + 2.0) * 2.0
    rel = 2.0 * R.sum_bound(v) + one + 8 * R.U32 * fin[:, None]
    away = torch.where(zo > -1e3, zo.abs(), zero)
    b_grad = q * (p.sum(dim=1) + p_t)[:, None] * (rel + 8 * R.U32 * z.abs()) \
        + p_t[:, None] * share * (rel + 8 * R.U32 * away) + share * one * tail \
        + pf * (one + 8 * R.U32 * lk.max(dim=1, keepdim=True).values) + 2.0 ** -126
    w = weight.double()[:, None] * scale
    return loss, grad * w, b_loss + 4 * R.U32 * loss.abs(), b_grad * w.abs()


def _check_all(x, k, scale, g):
    """Forward with and without lists and targets, its gradient, and distillation in both modes."""
    n, v = x.shape
    y = torch.randint(0, v, (n,), generator=g, device=DEV)
    r = _check_logprobs(x, y, k, scale)
    assert all(not torch.isnan(t).any() for t in r)
    _check_logprobs(x, None, 0, scale)
    gl, w = torch.randn(n, generator=g, device=DEV), torch.rand(n, generator=g, device=DEV) + 0.5
    ref, bound = R.logprobs_grad(x, y, gl, None, scale)
    d = B.tsid_token_logprobs_grad(x, y, r.row_max, r.log_sum, grad_logprob=gl, scale=scale)
    _within(d, ref, bound + R.stored(ref, x.dtype), "gradient")
    ids, lp = _teacher(x, k, g)
    for mode in (B.TSID_DISTILL_RENORM, B.TSID_DISTILL_TAIL):
        loss, grad, bl, bg = _distill(x, ids, lp, mode == B.TSID_DISTILL_TAIL, scale, w)
        for out_dtype in {torch.float32, x.dtype}:
            out = torch.empty(n, v, dtype=out_dtype, device=DEV)
            got = B.tsid_distill(x, ids, lp, mode=mode, scale=scale, weight=w, grad=out)
            _within(got, loss, bl, "loss")
            _within(out, grad, bg + R.stored(grad, out_dtype), "gradient of the loss")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("n,v", [(5, 4099), (2, 100_003), (460, 2051)])
def test_finite_scores_of_any_size(dtype, level, place, n, v):
    g = _gen(v + n)
    _check_all(_rows(place, level, n, v, dtype, g), 12, 1.0, g)


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("scale", [1e-20, 1e-6, 3e6, 3e8, 1e9, 1e12, 1e20])
@pytest.mark.parametrize("n,v", [(5, 4099), (2, 100_003), (460, 2051)])
def test_scores_at_any_accepted_scale(dtype, scale, n, v):
    g = _gen(v)
    _check_all((torch.randn(n, v, generator=g, device=DEV) * 2).to(dtype), 12, scale, g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", [(6, 3001), (3, 100_003), (460, 2051)])
def test_the_types_whole_range_at_the_smallest_scale(dtype, n, v):
    """Scores further apart than the type's largest value, which the scale brings back."""
    g = _gen(1)
    x = (torch.rand(n, v, generator=g, device=DEV) * 2 - 1) * 3.0e38
    x[1] = torch.finfo(dtype).min
    x[2, :2000] = torch.finfo(dtype).min
    _check_all(x.to(dtype), 8, 1e-20, g)
