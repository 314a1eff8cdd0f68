"""Attention over the paged cache where many rows share a key-value head, work that is taken in short runs, tables
past one CTA's shared memory, and references that move from tile to tile; against the same 64-bit formulas and bounds
as tests/test_gpu_kv.py."""
import random

import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R

import kv_util as K
from test_gpu_kv import BF16, DEV, F16, attend, check_attention, ints, make, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype,heads,kv_heads,page,lens,news,window", [
    (F16, 17, 1, 16, [1, 64, 65, 0, 300], [1, 1, 1, 0, 1], 0),            # one row past the narrow blocks
    (BF16, 32, 1, 8, [700, 5], [1, 1], 0),
    (F16, 64, 4, 64, [129, 400, 2], [4, 2, 1], 0),                        # 64 rows, 32, 16
    (BF16, 33, 1, 32, [500, 40], [2, 1], 0),                              # 66 rows
    (F16, 127, 1, 128, [333], [1], 0),
    (BF16, 128, 1, 64, [64, 1000], [1, 1], 0),
    (F16, 129, 1, 64, [200], [1], 0),                                     # a second block of one row
    (F16, 9, 3, 256, [600, 43, 64], [43, 43, 1], 0),                      # blocks that end inside a token's heads
    (BF16, 8, 2, 16, [64, 70, 1000], [64, 64, 33], 0),                    # a step as long as its sequence
    (F16, 40, 2, 32, [500, 90, 30], [3, 2, 1], 17),                       # sliding windows
    (BF16, 16, 1, 64, [300, 64], [20, 20], 64),
    (F16, 300, 1, 64, [90, 200], [2, 1], 0),                              # more heads than a block has rows
])
def test_wide_blocks(dim, dtype, heads, kv_heads, page, lens, news, window):
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, window=window, seed=heads)
    q = queries(kv, g)
    out = attend(kv, q)
    check_attention(kv, rows, lens, news, q, out, window=window)
    assert torch.equal(out, attend(kv, q))
    assert kv.stats()["status"] == B.LIF_OK
    kv.close()


@pytest.mark.parametrize("dim,heads,kv_heads,page,lens,new", [
    (128, 32, 4, 64, [9000, 2000, 777], 4),          # 32 rows: runs taken as CTAs become free
    (64, 71, 1, 64, [30000, 5000], 1),               # 71 rows: one run each
    (128, 16, 2, 8, [7000, 100], 64),                # 512 rows in four blocks, pages of 8
    (128, 8, 8, 32, [6000] * 12, 1),                 # narrow, long enough for short runs
    (80, 8, 2, 16, [20000, 3], 2),
    (256, 8, 2, 64, [9000, 500], 3)])
def test_many_launches_give_the_same_bits(dim, heads, kv_heads, page, lens, new):
    """Long sequences, launched over and over, eager and from a graph: whichever CTA takes a run, the output is the
    same, no wait runs out, and it is right."""
    news = [min(new, n) for n in lens]
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim, page=page)
    q = queries(kv, g)
    out = attend(kv, q)
    check_attention(kv, rows, lens, news, q, out)
    again = torch.full_like(q, 7)
    bad = torch.zeros((), dtype=torch.bool, device=DEV)
    for _ in range(100):
        again.fill_(7)
        kv.attention(0, q, out=again)
        bad |= (again != out).any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            kv.attention(0, q, out=again)
            bad |= (again != out).any()
    for _ in range(20):
        graph.replay()
    assert not bool(bad)
    assert kv.stats()["status"] == B.LIF_OK
    del graph
    kv.close()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window", [0, 20])
def test_what_is_not_seen_never_enters_a_wide_block(dtype, dim, window):
    """As for narrow blocks: infinities, NaN and the type's lowest value in rows that nobody sees, in the last token's
    row (which the tokens before it do not see), and in the first token's that leaves the window."""
    lens, news = [70, 64, 9, 140], [4, 3, 5, 1]
    kv, rows, g = make(lens, news, dtype=dtype, dim=dim, window=window, heads=20, kv_heads=2)
    q = queries(kv, g)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min], device=DEV).to(dtype)
    clean = kv.pages.clone()
    want = attend(kv, q)
    check_attention(kv, rows, lens, news, q, want, window=window)
    held = torch.zeros(kv.pages.shape[1], 16, dtype=torch.bool, device=DEV)
    for b, L in enumerate(lens):
        for p in range(max(0, L - news[b] + 1 - window) if window else 0, L):
            held[rows[b][p // 16], p % 16] = True
    fill = bad[torch.arange(kv.pages.numel(), device=DEV) % 4].view_as(kv.pages)
    kv.pages.copy_(torch.where(held[None, :, None, None, :, None], clean, fill))
    assert torch.equal(attend(kv, q), want)
    for b in range(len(lens)):
        p = lens[b] - 1
        kv.pages[0, rows[b][p // 16], :, :, p % 16] = fill[0, rows[b][p // 16], :, :, p % 16]
    out = attend(kv, q)
    for b, n in enumerate(news):
        u = K.U[dtype]
        # the same weights, the products formed one by one: fp32 sums of at most 140 terms in another order, and the
        # output's rounding on either side
        assert ((out[b, :n - 1].double() - want[b, :n - 1].double()).abs() <=
                2 * u * want[b, :n - 1].double().abs() + 2.0 ** -16).all()
        assert not torch.isfinite(out[b, n - 1]).all()
        assert (out[b, n:] == 7).all()
    kv.close()


@pytest.mark.parametrize("dim,heads,kv_heads,new", [(64, 4, 4, 1), (128, 8, 2, 2), (96, 6, 2, 3), (256, 4, 1, 2),
                                                    (64, 71, 1, 1), (128, 32, 2, 5)])
@pytest.mark.parametrize("slope", [0.05, -0.05, 3.0, -3.0])
def test_scores_that_rise_and_fall_along_the_sequence(dim, heads, kv_heads, new, slope):
    """Scores that climb (every tile moves the reference, by little or by more than a weight's range) or fall."""
    lens, news = [700, 150], [new, new]
    kv, rows, g = make(lens, news, heads=heads, kv_heads=kv_heads, dim=dim, page=16)
    q = queries(kv, g)
    q[..., 0] = 8.0
    scale = dim ** 0.5 / 8.0
    for b, L in enumerate(lens):
        at = torch.arange(L, device=DEV)
        page = torch.tensor(rows[b], device=DEV)[at // 16]
        # fp16 holds what is written; the oracle reads the same
        kv.pages[0, page, 0, :, at % 16, 0] = (slope * scale * (at - L / 2)).clamp(-60000, 60000).to(F16)[:, None].expand(-1, kv_heads)
    check_attention(kv, rows, lens, news, q, attend(kv, q))
    kv.close()


def test_tables_past_one_ctas_shared_memory():
    """A pool and a table that are handled by a cluster: random calls against the restatement."""
    rng = random.Random(9)
    max_seqs, page, n_pages, max_pages, max_new = 40, 8, 45000, 1700, 9
    pages = torch.zeros(1, n_pages, 2, 1, page, 64, device=DEV, dtype=F16)
    pages[..., 0] = torch.arange(n_pages, device=DEV).remainder(2048).half()[None, :, None, None, None]
    kv = R.KvCache(n_layers=1, n_heads=1, n_kv_heads=1, head_dim=64, n_pages=n_pages, max_seqs=max_seqs,
                   max_pages=max_pages, page_tokens=page, max_new=max_new, pages=pages)
    ref, mirror = K.Tables(max_seqs, max_pages, n_pages, page, max_new), pages.clone()
    order = list(range(n_pages))
    rng.shuffle(order)
    lens = [rng.choice([0, rng.randint(1, 300), rng.randint(6000, 8000)]) for _ in range(max_seqs)]
    rows, at = [], 0
    for n in lens:
        k = -(-n // page)
        rows.append(order[at:at + k])
        at += k
    table = ints([r + [-1] * (max_pages - len(r)) for r in rows])
    kv.load(ints(lens), table)
    ref.load(lens, rows, [0] * max_seqs)
    ref.check(kv)
    bad = table.clone()
    bad[lens.index(max(lens)), 3] = n_pages
    kv.load(ints(lens), bad)
    assert kv.stats()["status"] == B.LIF_ERR_INVALID_ARG
    ref.check(kv)
    kv.clear_status()
    for step in range(8):
        op = ["reserve", "fork", "compact", "reserve", "cut", "fork", "reserve", "compact"][step]
        copies = []
        if op == "reserve":
            n = [rng.choice([0, 1, rng.randint(0, max_new)]) for _ in range(max_seqs)]
            kv.reserve(ints(n))
            why, copies = ref.reserve(n)
            assert why is None
        elif op == "fork":
            src = [rng.choice([b, b, b, rng.randrange(max_seqs), -1]) for b in range(max_seqs)]
            kv.fork(ints(src))
            ref.fork(src)
        elif op == "cut":
            n = [rng.choice([-1, rng.randint(0, ref.lens[b])]) for b in range(max_seqs)]
            kv.fork(None, ints(n))
            ref.fork(None, n)
        else:
            kv.compact()
            copies = ref.compact()
        for s, d, r in copies:
            mirror[:, d, :, :, :r] = mirror[:, s, :, :, :r]
        ref.check(kv)
        assert torch.equal(mirror, kv.pages)
    kv.close()


def test_tables_of_ordinary_size_with_long_rows():
    """One CTA, rows of more pages than its warps hold in registers."""
    rng = random.Random(3)
    max_seqs, page, n_pages, max_pages = 5, 8, 30000, 9000
    kv = R.KvCache(n_layers=1, n_heads=1, n_kv_heads=1, head_dim=64, n_pages=n_pages, max_seqs=max_seqs,
                   max_pages=max_pages, page_tokens=page, max_new=2)
    ref = K.Tables(max_seqs, max_pages, n_pages, page, 2)
    order = list(range(n_pages))
    rng.shuffle(order)
    lens = [40000, 0, 70000, 5, 60001]
    rows, at = [], 0
    for n in lens:
        k = -(-n // page)
        rows.append(order[at:at + k])
        at += k
    kv.load(ints(lens), ints([r + [-1] * (max_pages - len(r)) for r in rows]), ints([1, 0, 2, 1, 2]))
    ref.load(lens, rows, [1, 0, 2, 1, 2])
    ref.check(kv)
    kv.fork(ints([2, 2, 0, 3, 4]), ints([-1, 5000, -1, -1, 30000]))
    ref.fork([2, 2, 0, 3, 4], [-1, 5000, -1, -1, 30000])
    ref.check(kv)
    kv.reserve(ints([1, 1, 2, 0, 1]))
    assert ref.reserve([1, 1, 2, 0, 1])[0] is None
    ref.check(kv)
    kv.compact()
    ref.compact()
    ref.check(kv)
    kv.close()


def test_norm_tensors_are_counted():
    kv = R.KvCache(n_layers=1, n_heads=4, n_kv_heads=4, head_dim=64, n_pages=4, max_seqs=1, norm=B.NORM_RMS)
    q = torch.zeros(1, 1, 4, 64, dtype=F16, device=DEV)
    w = torch.ones(64, dtype=F16, device=DEV)
    with pytest.raises(ValueError, match="norm tensors"):
        kv.append(0, q, q, q, norms=[w, w])
    kv.close()


def test_two_caches_with_wide_blocks_on_two_streams():
    """Their kernels take the tensor memory of the SMs in turn; a third stream's narrow cache runs beside them."""
    lens, news = [900, 90, 5000], [2, 1, 2]
    made = [make(lens, news, seed=s, dim=128, heads=h, kv_heads=2) for s, h in ((1, 32), (2, 64), (3, 4))]
    streams = [torch.cuda.Stream() for _ in made]
    qs = [queries(kv, g) for kv, _, g in made]
    outs = [torch.full_like(q, 7) for q in qs]
    torch.cuda.synchronize()
    for _ in range(30):
        for (kv, _, _), q, out, s in zip(made, qs, outs, streams):
            with torch.cuda.stream(s):
                kv.attention(0, q, out=out)
    for (kv, rows, _), q, out in zip(made, qs, outs):
        torch.cuda.synchronize()
        check_attention(kv, rows, lens, news, q, out)
        assert kv.stats()["status"] == B.LIF_OK
        kv.close()


def test_the_last_page_of_the_pool_and_of_a_sequence():
    """A reserve that takes every page, sequences that end at max_pages exactly, one token more refused; then attention
    over all of it, a fork that changes nothing but ends the step, and freeing."""
    page, max_pages, dim = 8, 4, 64
    kv = R.KvCache(n_layers=1, n_heads=4, n_kv_heads=2, head_dim=dim, n_pages=8, max_seqs=2, max_pages=max_pages,
                   page_tokens=page, max_new=32)
    ref = K.Tables(2, max_pages, 8, page, 32)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    kv.reserve(ints([32, 32]))
    assert ref.reserve([32, 32])[0] is None
    ref.check(kv)
    assert kv.stats()["free"] == 0
    q, k, v = queries(kv, g), queries(kv, g, 2), queries(kv, g, 2)
    kv.append(0, q, k, v, q_out=q)
    out = attend(kv, q)
    check_attention(kv, ref.rows, [32, 32], [32, 32], q, out)
    kv.fork()
    ref.fork()
    ref.check(kv)
    assert (attend(kv, q) == 7).all()                       # no step under way
    kv.reserve(ints([1, 0]))
    assert ref.reserve([1, 0])[0] == "capacity" and kv.stats()["status"] == B.LIF_ERR_CAPACITY
    ref.check(kv)
    kv.clear_status()
    kv.fork(ints([-1, 1]), ints([7, 25]))
    ref.fork([-1, 1], [7, 25])
    ref.check(kv)
    kv.reserve(ints([5, 7]))
    assert ref.reserve([5, 7])[0] is None
    ref.check(kv)
    out = attend(kv, q)
    check_attention(kv, ref.rows, [5, 32], [5, 7], q, out)
    kv.close()
