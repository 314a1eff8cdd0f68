"""Attention over long paged sequences: keys far below a row's largest weight, and every key counted once."""
import math

import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R

import kv_util as K
from test_gpu_kv import BF16, DEV, F16, attend, ints, make

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


@pytest.mark.parametrize("dim,dtype,heads,kv_heads,page,lens,new,window", [
    (64, F16, 4, 2, 64, [131001], 1, 0),
    (128, BF16, 32, 8, 128, [131001], 1, 0),
    (128, F16, 8, 8, 32, [6000] * 12, 1, 0),
    (128, F16, 56, 56, 32, [300 + 61 * i for i in range(64)], 1, 0),
    (80, F16, 8, 2, 16, [20000, 3, 777], 2, 0),
    (96, BF16, 12, 4, 32, [40000, 64, 1], 1, 0),
    (96, F16, 20, 1, 16, [9000, 130], 3, 0),
    (256, F16, 8, 2, 64, [30000, 500], 3, 0),
    (256, F16, 32, 2, 64, [9000, 65], 3, 0),
    (64, F16, 71, 1, 64, [30000, 5000], 1, 0),
    (64, F16, 71, 1, 64, [131001, 1, 64, 32000], 1, 0),
    (128, F16, 32, 4, 64, [9000, 2000, 777], 4, 0),
    (128, BF16, 16, 2, 8, [7000, 100], 64, 0),
    (128, F16, 64, 8, 64, [40000, 129], 16, 0),
    (64, F16, 4, 4, 64, [50000, 300], 2, 20000),
    (128, F16, 32, 2, 16, [50000, 300], 2, 20000),
])
def test_every_key_counts_once(dim, dtype, heads, kv_heads, page, lens, new, window):
    """Equal keys, so that all weights are one power of two, and values that say which tile of 64 keys they lie in: the
    first half of the columns by the tile's number modulo their count, the second half by the next digit of it.  The output
    is each column's share of the keys seen: a lost, doubled or exchanged piece of a tile shows.

    Bound, relative: the output's rounding u and 2^-19 for the exponentials (equal to one another; those of joined
    pieces 2^-22 off), the sums (multiples of one power of two, below 2^24 of it: exact) and the division."""
    news = [min(new, n) for n in lens]
    kv, rows, _ = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, window=window,
                       layer_values=False)
    half = dim // 2
    kv.pages.zero_()
    marks = []
    for b, L in enumerate(lens):
        at = torch.arange(L, device=DEV)
        tile = at // 64
        mark = torch.zeros(L, dim, device=DEV, dtype=torch.float64)
        mark[at, tile % half] = 1
        mark[at, half + tile // half % half] = 1
        pid = torch.tensor(rows[b], device=DEV)[at // page]
        kv.pages[0, pid, 1, :, at % page] = mark.to(dtype)[:, None].expand(-1, kv_heads, -1)
        marks.append(mark)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q = torch.randn(kv.max_seqs, kv.max_new, heads, dim, generator=g, device=DEV).to(dtype)
    out = attend(kv, q)
    u = K.U[dtype]
    for b, (L, n) in enumerate(zip(lens, news)):
        for t in range(n):
            p = L - n + t
            lo = max(0, p + 1 - window) if window else 0
            want = marks[b][lo:p + 1].mean(0)
            worst = ((out[b, t].double() - want).abs() - want * (u + 2.0 ** -19)).max()
            assert float(worst) <= 0, f"place {b}, token {t}"
        assert (out[b, n:] == 7).all()
    assert kv.stats()["status"] == B.LIF_OK
    kv.close()
