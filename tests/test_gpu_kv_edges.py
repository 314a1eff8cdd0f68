"""The paged key-value cache at its edges: scores far from zero, values that are not finite for every head dimension and
row count, calls that are refused, streams that are not the current one."""
import math

import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R

import kv_util as K
from test_gpu_kv import BF16, DEV, F16, attend, check_attention, ints, make, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 2, 2), (80, 8, 1), (96, 3, 3), (128, 2, 1), (256, 2, 2), (256, 20, 1),
                                                (64, 20, 1), (128, 20, 1)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("power,steps", [
    (24, [4, 8]), (24, [0, 4, 8, 12]), (24, [8, 4]), (26, [1, 3, 4]), (27, [1, 2]), (27, [0, 1]), (27, [2, 1, 3])])
def test_scores_far_from_zero(dim, heads, kv_heads, dtype, power, steps):
    """Scores of 2^power and a few units more (of the last place that fp32 has there), a tile of 64 keys for each of
    `steps`: the products and their sums are exact, the scale is ln 2, so that weights are powers of two of the
    differences, and no weight may leave fp16's range however the reference is rounded at that size.  The sequence stands in many
    places (all but their last pages are the same ones), so that runs hold several of its tiles.

    Bound: differences are multiples of 2 and at most 48, their product with scale log2(e) = 1 +- 2^-23 and the
    exponential are off by 48 2^-23 + 2^-21 relative (2^-17 covers both); the rest as in kv_util.attention."""
    tokens, page, unit, places, last = 64 * len(steps), 64, 2 ** (power - 23), 700, len(steps) - 1
    g = torch.Generator(device=DEV)
    g.manual_seed(dim + power)
    pages = torch.zeros(1, last + places, 2, kv_heads, page, dim, dtype=dtype, device=DEV)
    pages[0, :last + 1, 1].normal_(generator=g)
    pages[0, :, 0, :, :, 0] = 2.0 ** (power // 2)
    pages[0, :last + 1, 0, :, :, 1] = torch.tensor(steps, device=DEV, dtype=dtype)[:, None, None]
    pages[0, last + 1:] = pages[0, last]
    kv = R.KvCache(n_layers=1, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, n_pages=last + places, max_seqs=places,
                   max_pages=last + 1, page_tokens=page, dtype=dtype, pages=pages, scale=math.log(2.0))
    table = torch.arange(last + 1, dtype=torch.int32, device=DEV).repeat(places, 1)
    table[:, last] += torch.arange(places, dtype=torch.int32, device=DEV)
    kv.load(ints([tokens] * places), table, ints([1] * places))
    q = torch.zeros(places, 1, heads, dim, dtype=dtype, device=DEV)
    q[..., 0], q[..., 1] = 2.0 ** (power - power // 2), unit
    out = attend(kv, q)
    w = torch.tensor(steps, dtype=torch.float64, device=DEV).repeat_interleave(64) * unit
    w = torch.exp2(w - w.max())
    w = w / w.sum()
    V = K.held(pages, 0, list(range(len(steps))), tokens, 1)
    want = (w @ V).repeat_interleave(heads // kv_heads, 0)
    A = (w @ V.abs()).repeat_interleave(heads // kv_heads, 0)
    u, sub = K.U[dtype], 2.0 ** -32 if dtype == F16 else 0.0
    rel = u + 2.0 ** -17 + (tokens + 64) * 2.0 ** -23
    bound = u * want.abs() + rel * (1 + rel) * (A + want.abs()) + tokens * 2 * sub * V.abs().amax() + 2.0 ** -25
    assert torch.isfinite(out).all()
    worst = float(((out[:, 0].double() - want).abs() / bound).max())
    assert worst <= 1, f"{worst} of the bound"
    kv.close()


@pytest.mark.parametrize("max_seqs,n_pages,max_pages,per_place", [(5, 30000, 9000, 1500), (40, 45000, 1700, 1000)])
def test_bad_ids_behind_what_warps_hold_in_registers(max_seqs, n_pages, max_pages, per_place):
    """Tables handled by one CTA and by a cluster: a page id out of range among the pages of the step under way, in a
    chunk past those that stay in registers, is refused and changes nothing, whatever the scratch copy of the table held."""
    page = 8
    kv = R.KvCache(n_layers=1, n_heads=1, n_kv_heads=1, head_dim=64, n_pages=n_pages, max_seqs=max_seqs,
                   max_pages=max_pages, page_tokens=page, max_new=4)
    rows = [list(range(b * per_place, (b + 1) * per_place)) for b in range(max_seqs)]
    lens, news = [per_place * page - b % 3 for b in range(max_seqs)], [1 + b % 4 for b in range(max_seqs)]
    table = ints([r + [-1] * (max_pages - per_place) for r in rows])
    ref = K.Tables(max_seqs, max_pages, n_pages, page, 4)
    scratch = kv.workspace[kv.table.data_ptr() + 4 * kv.table.numel() - kv.workspace.data_ptr():
                           kv.refs.data_ptr() - kv.workspace.data_ptr()]
    assert scratch.numel() >= 4 * kv.table.numel()
    for loaded in (False, True):                             # into an empty cache, and over one that is in use
        if loaded:
            kv.clear_status()
            kv.load(ints(lens), table, ints(news))
            ref.load(lens, rows, news)
            assert kv.stats()["status"] == B.LIF_OK
            ref.check(kv)
        for b, j, bad in ((max_seqs - 1, per_place - 1, n_pages), (max_seqs - 1, per_place - 1, -1),
                          (max_seqs - 1, per_place - 1, 2 ** 31 - 1), (max_seqs - 2, 700, -2 ** 31), (max_seqs - 1, 40, n_pages)):
            wrong = table.clone()
            wrong[b, j] = bad
            scratch.fill_(0x7F)
            kv.clear_status()
            refused = kv.stats()["refused"]
            kv.load(ints(lens), wrong, ints(news))
            s = kv.stats()
            assert s["status"] == B.LIF_ERR_INVALID_ARG and s["refused"] == refused + 1
            ref.check(kv)
    kv.close()


@pytest.mark.parametrize("given", ["object", "number", "default", "none"])
def test_outputs_are_memory_of_the_stream_that_writes_them(given):
    """The current stream holds back a write into a block that the caller has dropped; a call on another stream that
    makes its own output may not be given that block."""
    lens, news = [70, 33], [2, 2]
    kv, rows, g = make(lens, news, heads=8, kv_heads=4, dim=128)
    q, k, v = queries(kv, g), queries(kv, g, 4), queries(kv, g, 4)
    side, busy = torch.cuda.Stream(), torch.cuda.Stream()
    stream = {"object": side, "number": side.cuda_stream, "default": 0, "none": None}[given]
    for call, right in ((lambda: kv.append(0, q, k, v, stream=stream), lambda out: torch.equal(out, q)),
                        (lambda: kv.attention(0, q, stream=stream),
                         lambda out: check_attention(kv, rows, lens, news, q, out) >= 0)):
        call()                                               # (no allocation from the device below)
        torch.cuda.synchronize()
        with torch.cuda.stream(busy):
            held = [torch.empty_like(q) for _ in range(4)]
            at = {t.data_ptr() for t in held}
            torch.cuda._sleep(20_000_000)                    # ten milliseconds
            for t in held:
                t.fill_(3)
            del held, t
            out = call()
            assert (out.data_ptr() in at) == (stream is None)     # the busy stream's own call may reuse its block
        torch.cuda.synchronize()
        assert right(out)
    assert kv.stats()["status"] == B.LIF_OK
    kv.close()


def test_attention_refuses_to_write_over_its_queries():
    kv, rows, g = make([40, 9], [2, 1], heads=4, kv_heads=2)
    q = queries(kv, g)
    n, was = q.numel(), q.clone()
    both = torch.zeros(3 * n, dtype=F16, device=DEV)
    at = lambda i: both[i:i + n].view_as(q)
    for a, b in ((q, q), (at(0), at(8)), (at(n - 8), at(0)), (at(n), at(8))):
        with pytest.raises(B.LifError) as e:
            kv.attention(0, a, out=b)
        assert e.value.code == B.LIF_ERR_INVALID_ARG
    assert torch.equal(q, was) and not both.any()
    for i, j in ((0, 1), (1, 0), (2, 1)):                    # side by side
        at(i * n).copy_(q)
        out = at(j * n).fill_(7)
        kv.attention(0, at(i * n), out=out)
        check_attention(kv, rows, [40, 9], [2, 1], q, out)
    assert kv.stats()["status"] == B.LIF_OK
    kv.close()


@pytest.mark.parametrize("max_seqs,max_new,heads,kv_heads", [(3, 2, 4, 2), (1, 1, 4, 4), (1, 3, 1, 1), (5, 1, 6, 3)])
def test_append_refuses_to_write_over_its_operands(max_seqs, max_new, heads, kv_heads):
    """All ways to lay queries, keys and values beside and over the block of queries that comes out; refused exactly
    where an element of theirs lies in it, unless the queries are that block."""
    dim, tokens = 64, max_seqs * max_new
    kv = R.KvCache(n_layers=1, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, n_pages=2 * max_seqs, max_seqs=max_seqs,
                   max_new=max_new, page_tokens=8)
    n, size = tokens * heads * dim, 24 * tokens * heads * dim
    block = torch.zeros(size, dtype=F16, device=DEV)
    base, out_at = block.data_ptr(), size // 2
    out = set(range(out_at, out_at + n, 8))
    far, seen = B.KvRows(base, 0, dim), set()                # n_heads * dim elements at most, at the beginning

    def rows_of(r, count):
        first = (r.dev - base) // 2
        return {first + t * r.token_stride + h * r.head_stride + e
                for t in range(tokens) for h in range(count) for e in range(0, dim, 8)}

    for token in (0, heads * dim, (heads + 2 * kv_heads) * dim, 3 * heads * dim, dim, 5 * n):
        for head in (dim, 3 * dim, tokens * dim, 0):
            for start in (out_at, out_at + n, out_at - dim, out_at + 8, out_at - 8, out_at + n - 8, out_at - token,
                          out_at - token * (tokens - 1) - head * (heads - 1) - dim, out_at - heads * dim, 0):
                start = max(0, start)
                for which, count in ((0, heads), (1, kv_heads), (2, kv_heads)):
                    r = B.KvRows(base + 2 * start, token, head)
                    if start + token * (tokens - 1) + head * (count - 1) + dim > size:
                        continue
                    packed = (tokens == 1 or token == heads * dim) and (heads == 1 or head == dim)
                    allowed = not rows_of(r, count) & out or (which == 0 and start == out_at and packed)
                    seen.add((which, allowed))
                    args = [far, far, far]
                    args[which] = r
                    if allowed:
                        B.lif_kv_append(kv.handle, 0, *args, None, base + 2 * out_at)
                    else:
                        with pytest.raises(B.LifError) as e:
                            B.lif_kv_append(kv.handle, 0, *args, None, base + 2 * out_at)
                        assert e.value.code == B.LIF_ERR_INVALID_ARG
    assert len(seen) == 6
    assert kv.stats()["status"] == B.LIF_OK and not block.any()          # (no step is under way: nothing was written)
    kv.close()


def _poison(kv):
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(kv.dtype).min], device=DEV).to(kv.dtype)
    return bad[torch.arange(kv.pages.numel(), device=DEV) % 4].view_as(kv.pages)


@pytest.mark.parametrize("dim,heads,kv_heads", [
    (64, 6, 3), (80, 4, 2), (96, 4, 2), (128, 4, 2), (256, 4, 2),         # up to 16 rows a key-value head
    (80, 8, 2), (96, 8, 2), (256, 8, 2),                                  # two tiles of rows,
    (80, 20, 2), (96, 20, 2), (256, 20, 2),                               # four,
    (80, 32, 2), (96, 32, 2), (256, 32, 2),                               # eight (256: two blocks of four)
    (80, 60, 2), (96, 60, 2),                                             # two blocks of eight
    (64, 32, 2), (64, 60, 2), (128, 32, 2), (128, 60, 2)])                # the tensor cores' blocks
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [0, 20])
def test_values_that_are_not_finite(dim, heads, kv_heads, dtype, window):
    """Infinities, NaN and the type's lowest value where no token sees them, then in the last token's row (which the tokens
    of its step before it do not see), then in the row that is the first token's last before it leaves the window (which the
    tokens behind it do not see): every token that does not see them as the formula has it, every one that does not finite."""
    lens, news = [70, 64, 9, 40, 200, 0], [4, 3, 5, 1, 2, 0]
    kv, rows, g = make(lens, news, dtype=dtype, dim=dim, heads=heads, kv_heads=kv_heads, window=window, seed=dim + heads)
    q = queries(kv, g)
    clean, fill = kv.pages.clone(), _poison(kv)
    want = attend(kv, q)
    check_attention(kv, rows, lens, news, q, want, window=window)
    first = [max(0, L - n + 1 - window) if window else 0 for L, n in zip(lens, news)]
    held = torch.zeros(kv.pages.shape[1], 16, dtype=torch.bool, device=DEV)
    for b, L in enumerate(lens):
        for p in range(first[b], L):
            held[rows[b][p // 16], p % 16] = True
    unseen = torch.where(held[None, :, None, None, :, None], clean, fill)

    def put(b, p):
        kv.pages[0, rows[b][p // 16], :, :, p % 16] = fill[0, rows[b][p // 16], :, :, p % 16]

    def check(out, b, t0, t1):
        """Tokens t0 .. t1-1 of place b."""
        if t1 > t0:
            y, bound = K.attention(q[b, t0:t1], clean, 0, rows[b], lens[b] - news[b] + t1, t1 - t0, window)
            assert ((out[b, t0:t1].double() - y).abs() <= bound).all()

    kv.pages.copy_(unseen)
    assert torch.equal(attend(kv, q), want)
    for b, L in enumerate(lens):
        if L:
            put(b, L - 1)
    out = attend(kv, q)
    for b, n in enumerate(news):
        check(out, b, 0, n - 1)
        assert n == 0 or not torch.isfinite(out[b, n - 1]).any()
        assert (out[b, n:] == 7).all()
    if window:
        kv.pages.copy_(unseen)
        leaves = [b for b, L in enumerate(lens) if L - news[b] + 1 > window]
        assert leaves
        for b in leaves:
            put(b, first[b])
        out = attend(kv, q)
        for b in leaves:
            check(out, b, 1, news[b])
            assert not torch.isfinite(out[b, 0]).any()
    assert kv.stats()["status"] == B.LIF_OK
    kv.close()


@pytest.mark.parametrize("dim,heads,kv_heads,max_new", [(64, 4, 2, 1), (128, 8, 1, 4), (80, 6, 2, 3)])
def test_few_places_in_use_far_apart(dim, heads, kv_heads, max_new):
    """1024 places of which a handful hold sequences, tables and attention."""
    live = {0: 90, 1: 7, 300: 700, 511: 64, 512: 65, 1000: 1, 1023: 333}
    lens = [live.get(b, 0) for b in range(1024)]
    news = [min(live.get(b, 0), max_new - b % 2 if max_new > 1 else 1) for b in range(1024)]
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim)
    q = queries(kv, g)
    check_attention(kv, rows, lens, news, q, attend(kv, q))
    kv.close()


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 8, 8), (128, 16, 2), (96, 8, 2), (256, 4, 2)])
def test_single_tokens_through_a_cache_for_pieces_of_a_prompt(dim, heads, kv_heads):
    """A prompt in steps of 64, a shorter last one, then single tokens: the same cache, every step's attention."""
    kv = R.KvCache(n_layers=1, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, n_pages=40, max_seqs=3, page_tokens=16,
                   max_new=64)
    g = torch.Generator(device=DEV)
    g.manual_seed(dim)
    ref = K.Tables(3, kv.max_pages, 40, 16, 64)
    for n in ([64, 64, 0], [64, 9, 40], [20, 1, 1], [1, 1, 1], [1, 0, 1], [1, 1, 5]):
        kv.reserve(ints(n))
        assert ref.reserve(n)[0] is None
        q, k, v = queries(kv, g), queries(kv, g, kv_heads), queries(kv, g, kv_heads)
        q2 = kv.append(0, q, k, v, q_out=torch.full_like(q, 7))
        for b in range(3):
            assert torch.equal(q2[b, :n[b]], q[b, :n[b]]) and (q2[b, n[b]:] == 7).all()
            if n[b]:
                for what, x in ((0, k), (1, v)):
                    got = K.held(kv.pages, 0, ref.rows[b], ref.lens[b], what)[:, ref.lens[b] - n[b]:]
                    assert torch.equal(got, x[b, :n[b]].transpose(0, 1).double())
        check_attention(kv, ref.rows, ref.lens, n, q, attend(kv, q))
    ref.check(kv)
    kv.close()
