"""The paged key-value cache on the GPU: tables against a plain restatement, appended rows and attention
against 64-bit formulas with derived bounds, refusals, values that must not be seen, streams, graphs,
and a token's run of append, attention and FFN layer-step together."""
import math
import random

import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R
from paper_2312_11514_b200 import workloads as W

import kv_util as K
import parity_util as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def make(lens, news, *, heads=4, kv_heads=4, dim=64, dtype=F16, page=16, layers=1, spare=3, seed=0, layer_values=True, **kw):
    """A cache whose places hold `lens` tokens (this step's `news` among them) on scattered pages."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    need = [-(-n // page) for n in lens]
    n_pages, width = sum(need) + spare, max(1, max(need))
    pages = torch.empty(layers, n_pages, 2, kv_heads, page, dim, dtype=dtype, device=DEV)
    if layer_values:
        pages.normal_(generator=g)
    order = torch.randperm(n_pages, generator=g, device=DEV).tolist()
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n])
        at += n
    kv = R.KvCache(n_layers=layers, n_heads=heads, n_kv_heads=kv_heads, head_dim=dim, n_pages=n_pages,
                   max_seqs=len(lens), max_pages=width, page_tokens=page, max_new=max(1, max(news)), dtype=dtype,
                   pages=pages, **kw)
    table = ints([r + [-1] * (width - len(r)) for r in rows])
    kv.load(ints(lens), table, ints(news))
    assert kv.stats()["status"] == B.LIF_OK
    return kv, rows, g


def queries(kv, g, heads=None):
    return torch.randn(kv.max_seqs, kv.max_new, heads or kv.n_heads, kv.head_dim, generator=g, device=DEV).to(kv.dtype)


def check_attention(kv, rows, lens, news, q, out, layer=0, window=0, scale=None):
    """All new tokens' outputs within their bounds, all other rows as they were (7)."""
    worst = 0.0
    for b, (L, n) in enumerate(zip(lens, news)):
        if n:
            want, bound = K.attention(q[b, :n], kv.pages, layer, rows[b], L, n, window, scale)
            diff = (out[b, :n].double() - want).abs()
            assert torch.isfinite(out[b, :n]).all()
            worst = max(worst, float((diff / bound).max()))
            assert (diff <= bound).all(), f"place {b}: {worst} of the bound"
        assert (out[b, n:] == 7).all(), f"place {b}: rows behind the step's tokens were written"
    return worst


def attend(kv, q, **kw):
    return kv.attention(0, q, out=torch.full_like(q, 7), **kw)


# ---- tables ---------------------------------------------------------------------------------------------


@pytest.mark.parametrize("max_seqs,page,n_pages,max_pages,max_new,seed", [
    (1, 8, 5, 4, 3, 0), (6, 8, 40, 6, 5, 1), (6, 16, 30, 9, 40, 2), (33, 8, 150, 7, 9, 3), (1024, 8, 5000, 5, 4, 4),
    (5, 256, 12, 3, 64, 5)])
def test_tables_follow_the_calls(max_seqs, page, n_pages, max_pages, max_new, seed):
    """Random reserves (some too large), forks, cuts, frees and compactions: tables, lengths, references,
    free pages and the pages' contents in every layer as the restatement has them."""
    rng = random.Random(seed)
    layers, dim, heads = 2, 64, 2
    pages = torch.randn(layers, n_pages, 2, heads, page, dim, device=DEV, dtype=F16)
    kv = R.KvCache(n_layers=layers, n_heads=heads, n_kv_heads=heads, head_dim=dim, n_pages=n_pages, max_seqs=max_seqs,
                   max_pages=max_pages, page_tokens=page, max_new=max_new, pages=pages)
    ref, mirror, refused = K.Tables(max_seqs, max_pages, n_pages, page, max_new), pages.clone(), 0
    seen = set()
    for step in range(40 if max_seqs < 100 else 12):
        op = rng.choice(["reserve", "reserve", "reserve", "fork", "cut", "compact"])
        if op == "reserve":
            n = [rng.choice([0, 1, 1, rng.randint(0, max_new)]) for _ in range(max_seqs)]
            if rng.random() < 0.1:
                n[rng.randrange(max_seqs)] = rng.choice([-1, max_new + 1])
            kv.reserve(ints(n))
            why, copies = ref.reserve(n)
        elif op == "fork":
            src = [rng.choice([b, b, rng.randrange(max_seqs), -1]) for b in range(max_seqs)]
            if rng.random() < 0.15:
                src[rng.randrange(max_seqs)] = rng.choice([-2, max_seqs])
            kv.fork(ints(src))
            why, copies = ref.fork(src), []
        elif op == "cut":
            src = list(range(max_seqs))
            if rng.random() < 0.5:
                rng.shuffle(src)
            n = [rng.choice([-1, rng.randint(0, ref.lens[s])]) for s in src]
            if rng.random() < 0.15:
                b = rng.randrange(max_seqs)
                n[b] = ref.lens[src[b]] + 1
            kv.fork(ints(src), ints(n))
            why, copies = ref.fork(src, n), []
        else:
            kv.compact()
            why, copies = None, ref.compact()
        for s, d, r in copies:
            mirror[:, d, :, :, :r] = mirror[:, s, :, :, :r]
        refused += why is not None
        seen.add((op, why, bool(copies)))
        ref.check(kv)
        assert torch.equal(mirror, kv.pages)
        assert kv.stats()["refused"] == refused
    if max_seqs == 6:
        assert len(seen) >= 6
    kv.close()


def test_copy_on_write_of_shared_pages():
    kv, rows, _ = make([21, 0, 0], [0, 0, 0], spare=8, layers=3)
    ref = K.Tables(3, kv.max_pages, kv.pages.shape[1], 16, 1)
    ref.load([21, 0, 0], [rows[0], [], []], [0, 0, 0])
    kv.fork(ints([0, 0, 0]), ints([21, 21, 18]))          # the third ends earlier in the same page
    ref.fork([0, 0, 0], [21, 21, 18])
    ref.check(kv)
    for n, copies in (([1, 1, 0], 2), ([1, 0, 1], 0)):    # the third holds on: both others copy; then nobody shares
        kv.reserve(ints(n))
        assert len(ref.reserve(n)[1]) == copies == kv.stats()["copies"]
        ref.check(kv)
    before = kv.pages.clone()
    kv.fork(ints([0, 0, 2]))
    ref.fork([0, 0, 2])
    kv.reserve(ints([1, 1, 1]))                            # all holders grow: the lowest keeps the page
    _, copies = ref.reserve([1, 1, 1])
    assert len(copies) == 1
    ref.check(kv)
    (s, d, r), = copies
    assert r == 23 % 16                                     # 21 tokens and two reserves
    before[:, d, :, :, :r] = before[:, s, :, :, :r]
    assert torch.equal(before, kv.pages)
    kv.close()


def test_refused_calls_change_nothing_and_are_recorded():
    kv, rows, g = make([30, 20, 5], [1, 1, 1], spare=1)
    ref = K.Tables(3, kv.max_pages, kv.pages.shape[1], 16, 1)
    ref.load([30, 20, 5], rows, [1, 1, 1])
    pages = kv.pages.clone()
    table, lens = kv.table.clone(), kv.lens.clone()
    for bad in (lambda: kv.fork(ints([0, 1, 3])), lambda: kv.fork(ints([0, 1, 2]), ints([31, 0, 0])),
                lambda: kv.fork(None, ints([-2, 0, 0])), lambda: kv.load(ints([30, 20, 33]), table),
                lambda: kv.load(ints([30, 20, -1]), table), lambda: kv.load(lens, table, ints([0, 2, 0])),
                lambda: kv.load(lens, ints([[0, kv.pages.shape[1]], [1, 2], [3, -1]])),
                lambda: kv.load(lens, ints([[0, -1], [1, 2], [3, -1]])),
                # page 0 of two places, one of which writes its step's token there
                lambda: kv.load(ints([30, 20, 5]), ints([[1, 0], [0, 2], [3, -1]]), ints([1, 0, 0]))):
        kv.clear_status()
        before = kv.stats()["refused"]
        bad()
        s = kv.stats()
        assert s["status"] == B.LIF_ERR_INVALID_ARG and s["refused"] == before + 1
        ref.check(kv)
    # shared, but not where the step's tokens lie
    kv.clear_status()
    kv.load(ints([30, 20, 5]), ints([[1, 0], [1, 2], [3, -1]]), ints([1, 1, 1]))
    assert kv.stats()["status"] == B.LIF_OK
    kv.load(lens, table)
    # capacity: one spare page, two wanted; then the step's calls do nothing
    kv.load(ints([32, 32, 5]), ints([[0, 1], [2, 3], [4, -1]]))
    kv.clear_status()
    kv.reserve(ints([1, 1, 1]))
    assert kv.stats()["status"] == B.LIF_ERR_CAPACITY
    assert kv.lens.tolist() == [32, 32, 5] and kv.n_new.tolist() == [0, 0, 0]
    q = queries(kv, g)
    kv.append(0, q, q, q, q_out=torch.full_like(q, 7))
    assert (attend(kv, q) == 7).all() and torch.equal(kv.pages, pages)
    # the first condition stands
    kv.fork(ints([9, 9, 9]))
    assert kv.stats()["status"] == B.LIF_ERR_CAPACITY
    kv.close()


def test_arguments_refused_on_the_host():
    kv, _, g = make([5], [1])
    q = queries(kv, g)
    big = torch.empty(q.numel() + 8, dtype=F16, device=DEV)
    for call, code in (
            (lambda: B.lif_kv_attention(kv.handle, 1, q, q), B.LIF_ERR_INVALID_ARG),
            (lambda: B.lif_kv_attention(kv.handle, -1, q, q), B.LIF_ERR_INVALID_ARG),
            (lambda: B.lif_kv_attention(kv.handle, 0, None, q), B.LIF_ERR_INVALID_ARG),
            (lambda: B.lif_kv_attention(kv.handle, 0, big.data_ptr() + 2, q), B.LIF_ERR_ALIGNMENT),
            (lambda: B.lif_kv_reserve(kv.handle, None), B.LIF_ERR_INVALID_ARG),
            (lambda: B.lif_kv_reserve(kv.handle, q.data_ptr() + 2), B.LIF_ERR_ALIGNMENT),
            (lambda: B.lif_kv_load(kv.handle, None, kv.table), B.LIF_ERR_INVALID_ARG)):
        with pytest.raises(B.LifError) as e:
            call()
        assert e.value.code == code
    good = B.KvRows(q.data_ptr(), 256, 64)
    for bad, code in ((B.KvRows(q.data_ptr(), 252, 64), B.LIF_ERR_ALIGNMENT), (B.KvRows(q.data_ptr(), 256, 4), B.LIF_ERR_ALIGNMENT),
                      (B.KvRows(q.data_ptr() + 8, 256, 64), B.LIF_ERR_ALIGNMENT), (B.KvRows(None, 256, 64), B.LIF_ERR_INVALID_ARG),
                      (B.KvRows(q.data_ptr(), -256, 64), B.LIF_ERR_INVALID_ARG)):
        for args in ((bad, good, good), (good, bad, good), (good, good, bad)):
            with pytest.raises(B.LifError) as e:
                B.lif_kv_append(kv.handle, 0, *args, None, q)
            assert e.value.code == code
    for t in (q[:, :, :2], q.float(), q.cpu(), q.transpose(2, 3)):
        with pytest.raises(ValueError):
            kv.attention(0, t)
    with pytest.raises(ValueError):
        kv.reserve(torch.zeros(1, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        R.KvCache(n_layers=1, n_heads=4, n_kv_heads=4, head_dim=64, n_pages=4, max_seqs=1, dtype=torch.float32)
    kv.close()
    normed = R.KvCache(n_layers=1, n_heads=4, n_kv_heads=4, head_dim=64, n_pages=4, max_seqs=1, norm=B.NORM_RMS)
    q = queries(normed, g)
    with pytest.raises(B.LifError) as e:
        normed.append(0, q, q, q)                            # weights are missing
    assert e.value.code == B.LIF_ERR_INVALID_ARG
    normed.close()


# ---- append -----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,dtype,heads,kv_heads,page,new,norm,rope,dims,base,fused", [
    (64, F16, 4, 4, 16, 1, 0, 0, 0, 1e4, False),
    (64, F16, 64, 64, 16, 1, 2, 1, 32, 25e3, True),
    (80, F16, 32, 32, 64, 5, 0, 1, 32, 1e4, True),
    (80, BF16, 5, 5, 8, 3, 1, 1, 40, 1e4, False),           # pairs 20 apart
    (96, F16, 6, 2, 32, 7, 2, 2, 96, 1e6, True),
    (96, BF16, 3, 3, 16, 2, 1, 1, 90, 1e4, False),          # pairs 45 apart
    (128, BF16, 32, 8, 128, 64, 1, 2, 128, 1e4, True),
    (128, F16, 2, 1, 8, 1, 2, 1, 2, 1e4, False),            # one pair
    (256, F16, 8, 1, 256, 3, 1, 1, 256, 1e6, True),
    (256, BF16, 2, 2, 16, 9, 2, 2, 50, 1e4, False)])
def test_append(dim, dtype, heads, kv_heads, page, new, norm, rope, dims, base, fused):
    lens, news = [page + 3, 0, new, 2 * page, 1000 + new], [new, 0, new, max(1, new - 1), 1]
    lens[3] = max(lens[3], new)
    freq = R.rope_frequencies(dims, base) if rope else None
    lens[0] = max(lens[0], new)
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, layers=2,
                       norm=norm, norm_eps=1e-5, rope=rope, rope_dims=dims, rope_freq=freq, rope_scale=1.125)
    if fused:
        x = queries(kv, g, heads + 2 * kv_heads) * 3
        q, k, v = x[:, :, :heads], x[:, :, heads:heads + kv_heads], x[:, :, heads + kv_heads:]
    else:
        q, k, v = queries(kv, g) * 3, queries(kv, g, kv_heads) * 3 + 1, queries(kv, g, kv_heads)
    w = [1 + 0.3 * torch.randn(dim, generator=g, device=DEV) for _ in range(4)]
    w = [t.to(dtype) for t in w]
    if norm == B.NORM_RMS:
        w[1] = w[3] = None
    before = kv.pages.clone()
    want = before.double()
    slack = torch.zeros_like(want)
    got = kv.append(1, q, k, v, q_out=torch.full((len(lens), kv.max_new, heads, dim), 7.0, dtype=dtype, device=DEV),
                    norms=w if norm else None)
    for b, (L, n) in enumerate(zip(lens, news)):
        for t in range(n):
            pos = L - n + t
            y, bound = K.rotated(q[b, t], pos, norm, w[0], w[1], 1e-5, rope, dims, freq, 1.125)
            assert ((got[b, t].double() - y).abs() <= bound).all()
            y, bound = K.rotated(k[b, t], pos, norm, w[2], w[3], 1e-5, rope, dims, freq, 1.125)
            page_id = rows[b][pos // page]
            want[1, page_id, 0, :, pos % page], slack[1, page_id, 0, :, pos % page] = y, bound
            want[1, page_id, 1, :, pos % page] = v[b, t].double()
        assert (got[b, n:] == 7).all()
    assert ((kv.pages.double() - want).abs() <= slack).all()
    kv.close()


def test_append_far_positions_and_queries_in_place():
    """Angles at positions where an fp32 product is off by radians; the pages before are one shared page."""
    n, far, freq = 4, (1 << 22) - 1, R.rope_frequencies(64, 1e4)
    kv = R.KvCache(n_layers=1, n_heads=2, n_kv_heads=1, head_dim=64, n_pages=3, max_seqs=1, max_pages=1 << 14,
                   page_tokens=256, max_new=n, rope=B.ROPE_HALF, rope_dims=64, rope_freq=freq)
    table = torch.zeros(1, 1 << 14, dtype=torch.int32, device=DEV)
    table[0, -1] = 2
    kv.load(ints([far]), table, ints([n]))
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q, k = queries(kv, g), queries(kv, g, 1)
    was = q.clone()
    kv.append(0, q, k, k, q_out=q)
    for t in range(n):
        y, bound = K.rotated(was[0, t], far - n + t, 0, None, None, 0, 1, 64, freq, 1.0)
        assert ((q[0, t].double() - y).abs() <= bound).all()
        y, bound = K.rotated(k[0, t], far - n + t, 0, None, None, 0, 1, 64, freq, 1.0)
        row = (far - n + t) % 256
        assert ((kv.pages[0, 2, 0, :, row].double() - y).abs() <= bound).all()
        assert torch.equal(kv.pages[0, 2, 1, :, row], k[0, t])
    kv.close()


# ---- attention ----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dim", [64, 80, 96, 128, 256])
@pytest.mark.parametrize("dtype,heads,kv_heads,page,lens,news,window", [
    (F16, 4, 4, 16, [1], [1], 0),                                     # one token, itself only
    (F16, 4, 4, 16, [1, 63, 64, 65, 127, 128, 129, 0], [1] * 7 + [0], 0),
    (BF16, 3, 3, 8, [200, 5, 0, 77], [5, 5, 0, 1], 0),                # several tokens, some at the very beginning
    (F16, 6, 2, 256, [700, 64, 300], [3, 8, 1], 0),                   # two row tiles
    (BF16, 8, 1, 32, [513, 90], [7, 2], 0),                           # four
    (F16, 71, 1, 64, [1000, 17, 4000], [1, 1, 1], 0),                 # five of eight
    (F16, 20, 1, 64, [640, 700], [16, 9], 0),                         # several row blocks
    (F16, 2, 2, 64, [300, 64, 65], [64, 64, 64], 0),                  # longest steps
    (F16, 4, 4, 16, [500, 20, 64], [1, 1, 1], 16),                    # sliding windows
    (BF16, 4, 2, 32, [500, 40, 129], [6, 40, 20], 33),
    (F16, 4, 4, 16, [100, 30], [3, 2], 1),                            # only itself
])
def test_attention(dim, dtype, heads, kv_heads, page, lens, news, window):
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, window=window, seed=dim)
    q = queries(kv, g)
    out = attend(kv, q)
    check_attention(kv, rows, lens, news, q, out, window=window)
    assert torch.equal(out, attend(kv, q))                             # the same bits again
    kv.close()


@pytest.mark.parametrize("heads,kv_heads,lens,new", [
    (32, 32, [9000], 1), (8, 2, [40000, 3], 1), (71, 1, [30000], 1), (32, 8, [12000, 500], 5)])
def test_attention_over_long_sequences_is_split_and_joined(heads, kv_heads, lens, new):
    news = [min(new, n) for n in lens]
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=128 if kv_heads > 1 else 64, page=64)
    q = queries(kv, g) * 4                                             # weights that differ
    check_attention(kv, rows, lens, news, q, attend(kv, q))
    kv.close()


def test_attention_many_ragged_sequences():
    rng = random.Random(5)
    lens = [rng.choice([0, 1, rng.randint(1, 600)]) for _ in range(200)]
    news = [min(n, rng.randint(0, 2)) for n in lens]
    kv, rows, g = make(lens, news, heads=2, kv_heads=2, dim=64, page=16)
    q = queries(kv, g)
    check_attention(kv, rows, lens, news, q, attend(kv, q))
    kv.close()


def test_attention_scale_and_second_layer():
    kv, rows, g = make([77, 130], [2, 1], layers=3, scale=0.25, dim=80)
    q = queries(kv, g)
    out = kv.attention(2, q, out=torch.full_like(q, 7))
    check_attention(kv, rows, [77, 130], [2, 1], q, out, layer=2, scale=0.25)
    kv.close()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [0, 20])
def test_what_is_not_seen_never_enters(dtype, window):
    """Infinities, NaN and the type's extremes in keys and values that a token does not see: the free rows of
    the last page, other pages, later tokens of the step, tokens that have left the window."""
    lens, news = [70, 64, 9, 40], [4, 3, 5, 1]
    kv, rows, g = make(lens, news, dtype=dtype, window=window, heads=4, kv_heads=2)
    q = queries(kv, g)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min], device=DEV).to(dtype)
    clean = kv.pages.clone()
    want = attend(kv, q)
    check_attention(kv, rows, lens, news, q, want, window=window)
    held = torch.zeros(kv.pages.shape[1], 16, dtype=torch.bool, device=DEV)
    for b, L in enumerate(lens):
        first = max(0, L - news[b] + 1 - window) if window else 0
        for p in range(first, L):
            held[rows[b][p // 16], p % 16] = True
    fill = bad[torch.arange(kv.pages.numel(), device=DEV) % 4].view_as(kv.pages)
    kv.pages.copy_(torch.where(held[None, :, None, None, :, None], clean, fill))
    assert torch.equal(attend(kv, q), want)                            # unheld and unseen rows
    for b in range(len(lens)):                                         # the last token's own row
        p = lens[b] - 1
        kv.pages[0, rows[b][p // 16], :, :, p % 16] = fill[0, rows[b][p // 16], :, :, p % 16]
    out = attend(kv, q)
    for b, n in enumerate(news):
        u = K.U[dtype]
        # the earlier tokens of the step: the same sums, the values' products formed one by one
        assert ((out[b, :n - 1].double() - want[b, :n - 1].double()).abs() <=
                2 * u * want[b, :n - 1].double().abs() + 2.0 ** -16).all()
        assert not torch.isfinite(out[b, n - 1]).all()
    if window:                                                         # the first seen token's row leaves the window
        kv.pages.copy_(torch.where(held[None, :, None, None, :, None], clean, fill))
        for b, L in enumerate(lens):
            p = max(0, L - news[b] + 1 - window)
            if L > news[b] + window:
                kv.pages[0, rows[b][p // 16], :, :, p % 16] = fill[0, rows[b][p // 16], :, :, p % 16]
                out = attend(kv, q)
                assert ((out[b, 1:news[b]].double() - want[b, 1:news[b]].double()).abs() <=
                        2 * K.U[dtype] * want[b, 1:news[b]].double().abs() + 2.0 ** -16).all()
    kv.close()


def test_extreme_scores():
    """One key far above the rest, equal keys, and scores of either sign's largest finite products."""
    kv, rows, g = make([200, 130], [1, 1], heads=2, kv_heads=1)
    q = queries(kv, g)
    q[:, :, 0] = 200.0
    q[:, :, 1] = -200.0
    kv.pages[0, rows[0][3], 0, :, 5] = 300.0                            # score 480000 and -480000
    kv.pages[0, rows[1][0], 0, :, :] = -300.0
    check_attention(kv, rows, [200, 130], [1, 1], q, attend(kv, q))
    kv.pages[0, :, 0] = 1.0                                             # all weights alike: the mean of the values
    check_attention(kv, rows, [200, 130], [1, 1], q, attend(kv, q))
    kv.close()


def test_large_pool_offsets():
    """A pool past 2^31 elements (and 2^32 bytes): pages on both sides, in the last layer."""
    n_pages, page, kvh, dim = 4200, 256, 4, 128
    pages = torch.empty(2, n_pages, 2, kvh, page, dim, dtype=F16, device=DEV)
    assert pages[0].numel() > 2 ** 30 and pages.numel() > 2 ** 31
    rows = [[n_pages - 1, 0, n_pages - 2], [4096, 4095]]
    pages[1, [r for row in rows for r in row]] = torch.randn(5, 2, kvh, page, dim, device=DEV).half()
    kv = R.KvCache(n_layers=2, n_heads=4, n_kv_heads=kvh, head_dim=dim, n_pages=n_pages, max_seqs=2, max_pages=3,
                   page_tokens=page, max_new=2, pages=pages)
    kv.load(ints([600, 300]), ints([rows[0], rows[1] + [-1]]), ints([2, 1]))
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    q, k, v = queries(kv, g), queries(kv, g), queries(kv, g)
    q2 = kv.append(1, q, k, v)
    assert torch.equal(kv.pages[1, n_pages - 2, 1, :, 599 - 512], v[0, 1])
    out = kv.attention(1, q, out=torch.full_like(q, 7))
    check_attention(kv, rows, [600, 300], [2, 1], q, out, layer=1)
    assert torch.equal(q2[0], q[0])
    kv.compact()                                                        # every page from the far end to the beginning
    torch.cuda.synchronize()
    assert sorted(kv.table[kv.table >= 0].tolist()) == [0, 1, 2, 3, 4]
    assert torch.equal(kv.attention(1, q, out=torch.full_like(q, 7)), out)
    kv.close()


# ---- together -------------------------------------------------------------------------------------------------


def test_other_streams_and_two_caches_at_once():
    made = [make([400, 90, 3], [2, 1, 3], seed=s, dim=128, heads=8, kv_heads=4) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in made]
    qs = [queries(kv, g) for kv, _, g in made]
    outs = [torch.full_like(q, 7) for q in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for (kv, _, _), q, out, s in zip(made, qs, outs, streams):
            with torch.cuda.stream(s):
                kv.attention(0, q, out=out)
    for (kv, rows, _), q, out in zip(made, qs, outs):
        torch.cuda.synchronize()
        check_attention(kv, rows, [400, 90, 3], [2, 1, 3], q, out)
        kv.close()


def _program(kv, layers, wq, wo, sc):
    """One token as a program runs it: per layer projection, append, attention, projection, FFN layer-step."""
    S, H, D = kv.max_seqs, kv.n_heads, kv.head_dim
    x = torch.zeros(S, H * D, dtype=F16, device=DEV)
    n_new = torch.ones(S, dtype=torch.int32, device=DEV)
    ys = torch.zeros(len(layers), S, H * D, dtype=torch.float32, device=DEV)
    q_out = torch.zeros(S, 1, H, D, dtype=F16, device=DEV)
    att = torch.zeros(len(layers), S, 1, H, D, dtype=F16, device=DEV)

    def token():
        kv.reserve(n_new)
        h = x
        for l, layer in enumerate(layers):
            qkv = (h @ wq[l]).view(S, 1, 3 * H, D)
            kv.append(l, qkv[:, :, :H], qkv[:, :, H:2 * H], qkv[:, :, 2 * H:], q_out=q_out)
            kv.attention(l, q_out, out=att[l])
            h = h + att[l].view(S, H * D) @ wo[l]
            B.lif_decode_step(layer.handle, h, ys[l], sc, sc)
            h = (h + 0.1 * ys[l].half())
        return h

    return x, token, att, ys


def test_tokens_through_attention_and_ffn_eager_and_as_a_graph():
    """Two layers over several tokens, eager and as one captured graph that is replayed: the same outputs, and the
    attention of the last token as the formula has it; then drafts are dropped and a sequence is copied, and the graph
    goes on."""
    cfg = W.CONFIGS["tiny"].scaled(n_streams=2, mean_fire=0.1)
    S, H, D = 2, 4, 64
    freq = R.rope_frequencies(32)

    def build():
        layers = R.build_stack(cfg, device=DEV, capacity_margin=30.0)
        kv = R.KvCache(n_layers=2, n_heads=H, n_kv_heads=H, head_dim=D, n_pages=24, max_seqs=S, page_tokens=8,
                       rope=B.ROPE_HALF, rope_dims=32, rope_freq=freq)
        g = torch.Generator(device=DEV)
        g.manual_seed(11)
        wq = torch.randn(2, H * D, 3 * H * D, generator=g, device=DEV).half() * 0.06
        wo = torch.randn(2, H * D, H * D, generator=g, device=DEV).half() * 0.06
        return layers, kv, wq, wo

    xs = W.make_inputs(cfg, device=DEV)
    results = []
    for captured in (False, True):
        layers, kv, wq, wo = build()
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            x, token, att, ys = _program(kv, layers, wq, wo, s)
            kv.pages.zero_()
            token()                                       # warm-up (allocations, library handles)
            kv.reset()
            for layer in layers:
                B.lif_reset(layer.handle, s)
            torch.cuda.synchronize()
            run = token
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=s):
                    token()
                run = graph.replay
            seen = []
            for t in range(20):
                x.copy_(xs[t % xs.shape[0]])
                run()
                seen.append((att.clone(), ys.clone()))
                if t == 11:
                    kv.fork(None, ints([9, -1]))          # three tokens of the first sequence are dropped
                if t == 14:
                    kv.fork(ints([1, 1]))                 # both go on from the second
            torch.cuda.synchronize()
        st = kv.stats()
        assert st["status"] == B.LIF_OK
        assert kv.lens.tolist() == [20, 20]
        results.append((seen, kv.table.cpu(), kv.pages.clone()))
        del run
        if captured:
            del graph
        kv.close()
        for layer in layers:
            assert B.lif_get_stats(layer.handle).status == B.LIF_OK
            layer.close()
    (eager, table, pages), (graph, table2, pages2) = results
    assert torch.equal(table, table2) and torch.equal(pages, pages2)
    for (a, y), (a2, y2) in zip(eager, graph):
        assert torch.equal(a, a2) and torch.equal(y, y2)
