"""Attention over long paged sequences: keys far below a row's largest weight."""
import math

import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R

import kv_util as K
from test_gpu_kv import BF16, DEV, F16, attend, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,heads,kv_heads,dtype,at,tokens", [
    (64, 2, 2, F16, 5, 131001),
    (80, 4, 1, F16, 70003, 131001),
    (96, 2, 1, F16, 5, 131001),
    (128, 2, 2, F16, 40, 131001),
    (128, 2, 2, BF16, 40, 131001),
    (256, 1, 1, F16, 5, 131001),
    (64, 20, 1, F16, 5, 131001),                     # row blocks of the tensor cores' 128
    (128, 20, 1, F16, 70003, 131001),
    (128, 20, 1, BF16, 5, 131001),
    (64, 1, 1, F16, 5, 1 << 20),
])
def test_many_keys_far_below_the_largest(dim, heads, kv_heads, dtype, at, tokens):
    """One key that nearly all the weight goes to and whose value is nothing, and a long sequence of weights around
    2^-25.5 of it: together they are a few thousandths, and all of the output.  The sequence stands in as many places
    as there are CTAs (all but their last pages are the same ones), so that a run holds most of it.

    Bound, relative to the output (all values are positive, so what a weight is off by moves the output by as much at
    most): the score's sum and the exponential as in kv_util.attention, a weight's rounding u, the fp32 sums' (tokens +
    64) 2^-23, the output's rounding u.  Where a weight is below the normal numbers of fp16 its rounding is absolute:
    2^-25 of what is 2^7 for the largest weight (at least), 2^-32 for each key and value of 1.5 at most."""
    places, page = 300, 64
    shared = -(-tokens // page) - 1
    g = torch.Generator(device=DEV)
    g.manual_seed(dim)
    pages = torch.zeros(1, shared + places, 2, kv_heads, page, dim, dtype=dtype, device=DEV)
    # log2 of a weight: -25.25 and less by sixteenths (scores whose products and sums are exact in either type)
    falls = torch.randint(0, 8, (shared + 1, kv_heads, page), generator=g, device=DEV) / 16
    pages[0, :shared + 1, 0, :, :, 0] = -falls.to(dtype)
    pages[0, :shared + 1, 1] = (torch.rand(shared + 1, kv_heads, page, dim, generator=g, device=DEV) + 0.5).to(dtype)
    pages[0, at // page, 0, :, at % page, 0] = 0
    pages[0, at // page, 0, :, at % page, 1] = 1
    pages[0, at // page, 1, :, at % page] = 0
    pages[0, shared + 1:] = pages[0, shared]
    scale = math.log(2.0)
    kv = R.KvCache(n_layers=1, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, n_pages=shared + places, max_seqs=places,
                   max_pages=shared + 1, page_tokens=page, dtype=dtype, pages=pages, scale=scale)
    table = torch.arange(shared + 1, dtype=torch.int32, device=DEV).repeat(places, 1)
    table[:, shared] += torch.arange(places, dtype=torch.int32, device=DEV)
    kv.load(ints([tokens] * places), table, ints([1] * places))
    q = torch.zeros(places, 1, heads, dim, dtype=dtype, device=DEV)
    q[..., 0], q[..., 1] = 1.0, 25.25
    out = attend(kv, q)
    assert kv.stats()["status"] == B.LIF_OK
    want, _ = K.attention(q[0], pages, 0, list(range(shared + 1)), tokens, 1, scale=scale)
    u, absolute = K.U[dtype], tokens * 1.5 * 2.0 ** -32 if dtype == F16 else 0.0
    rel = u + (dim + 8) * 2.0 ** -23 * scale * 25.25 + 2.0 ** -17 + (tokens + 64) * 2.0 ** -23
    bound = want * (u + rel * (1 + rel)) + absolute
    worst = float(((out.double() - want).abs() / bound).max())
    assert worst <= 1, f"{worst} of the bound"
    kv.close()
