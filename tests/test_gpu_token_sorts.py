"""Gradient of the lookup: every form of the sort at its borders, digits of large tables, accumulation, and types and
strides of large batches."""
import pytest
import torch

import token_reference as R
from paper_2608_00977_b200 import binding as B
from test_gpu_token_ops import DEV, _gen, _ids, _place, _put, _within

pytestmark = pytest.mark.gpu


def _check(dy, ids, rows, out_dtype, pad=0, shift=0, accumulate=False, g=None):
    dim = dy.shape[1]
    ref, bound = R.embed_grad(dy, ids, rows, 0.5)
    out = _place(rows, dim, out_dtype, pad, shift)
    if accumulate:
        out.copy_(torch.randn(rows, dim, generator=g, device=DEV))
        ref = ref + out.double()          # one multiply-add of the sum in fp32, then the store
    else:
        out.fill_(float("nan"))
    old = out.clone()
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tsid_embed_grad(dy, ids, rows, scale=0.5, out=out, accumulate=accumulate, flag=flag)
    _within(out, ref, bound + R.stored(ref, out_dtype), "gradient")
    assert flag.item() == 0
    if accumulate:                        # rows that no id names are left alone, bit for bit
        other = torch.ones(rows, dtype=torch.bool, device=DEV)
        other[ids[ids >= 0].long()] = False
        assert torch.equal(out[other], old[other])


@pytest.mark.parametrize("tokens", [256, 257, 1024, 1025, 16_383, 16_384, 16_385, 32_767, 32_768, 32_769, 65_535, 65_537])
@pytest.mark.parametrize("kind,rows", [("uniform", 5000), ("skewed", 500), ("uniform", 2 ** 18 - 1), ("uniform", 2 ** 18), ("one", 2 ** 18 + 3)])
def test_the_sorts_at_their_borders(tokens, kind, rows):
    """One, two and four items a thread, up to 16 CTAs; two digits below 2^18 rows and three from there."""
    g = _gen(tokens + rows)
    dy = torch.randn(tokens, 16, generator=g, device=DEV).bfloat16()
    _check(dy, _ids(kind, tokens, rows, g), rows, torch.float32)


@pytest.mark.parametrize("rows", [1, 2, 1023, 1024, 2 ** 20 - 1, 2 ** 20, 2_000_000])
@pytest.mark.parametrize("kind", ["uniform", "skewed", "each"])
def test_digits_of_large_batches(rows, kind):
    """Digits of up to ten bits: one below 1,024 rows, two below 2^20, three from there."""
    g = _gen(rows)
    dy = torch.randn(100_003, 8, generator=g, device=DEV)
    _check(dy, _ids(kind, 100_003, rows, g), rows, torch.float32)


@pytest.mark.parametrize("tokens,rows", [(7, 2 ** 24), (256, 2 ** 24 + 5)])
def test_a_small_batch_on_a_table_of_more_than_2_24_rows(tokens, rows):
    g = _gen(tokens)
    ids = torch.randint(0, rows, (tokens,), generator=g, device=DEV)
    ids[0] = rows - 1
    _check(torch.randn(tokens, 3, generator=g, device=DEV), ids, rows, torch.bfloat16)


@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in R.DTYPES for b in R.DTYPES])
@pytest.mark.parametrize("kind,tokens,rows,dim,pad,shift", [
    ("uniform", 40, 300, 24, 0, 0), ("skewed", 250, 40, 33, 2, 1), ("skewed", 3000, 400, 64, 8, 0), ("uniform", 20_000, 3000, 40, 0, 0),
    ("skewed", 70_001, 4000, 32, 0, 0), ("uniform", 120_000, 50_000, 17, 3, 1), ("one", 66_000, 9, 64, 4, 2)])
def test_accumulation_and_strided_tables(dtype, out_dtype, kind, tokens, rows, dim, pad, shift):
    g = _gen(tokens + dim)
    dy = _put(torch.randn(tokens, dim, generator=g, device=DEV).to(dtype), pad, shift)
    ids = _ids(kind, tokens, rows, g)
    _check(dy, ids, rows, out_dtype, pad, shift)
    _check(dy, ids, rows, out_dtype, pad, shift, accumulate=True, g=g)


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,v", [(74, 100_000), (90, 60_001), (60, 150_003)])
def test_distillation_with_nine_to_fifteen_ctas_a_row(dtype, tail, n, v):
    from test_gpu_token_ops import _teacher
    g = _gen(n)
    x = (torch.randn(n, v, generator=g, device=DEV) * 2).to(dtype)
    ids, lp = _teacher(x, 30, g)
    loss, grad, bl, bg = R.distill(x, ids, lp, tail, 1.0)
    out = torch.empty_like(x)
    got = B.tsid_distill(x, ids, lp, mode=B.TSID_DISTILL_TAIL if tail else B.TSID_DISTILL_RENORM, grad=out)
    _within(got, loss, bl + 4 * R.U32 * loss.abs(), "loss")
    _within(out, grad, bg + R.stored(grad, dtype), "gradient")
