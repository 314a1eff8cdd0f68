"""The attention side of a decoded token, measured: what stands between two FFN layer-steps.

A case names the heads (`heads`, `kv_heads`, `dim`), the type, the page size in tokens and the
sequences: `seqs` places, whose lengths are spread over `len_min` .. `len_max` (by the logarithm;
the same for every seed), `new` tokens each in this step (`ragged`: some fewer, some places
empty).  `op` is what a pass does:

  append  norm of queries and keys per head, rotation of positions, keys and values into their pages
  attend  attention of the new tokens over the cached ones
  grow    every sequence becomes `fan` copies of itself (pages shared), then takes `new` tokens:
          pages are given out, and a partly filled page that is shared is copied
  compact pages scattered over the pool move to its beginning, tables and all

All passes can be repeated: `append` writes the same places again, `grow` starts by cutting the
sequences back to the lengths that they had, `compact` by loading the scattered tables."""
import math
import random

import torch

own = False

NORM_NONE, NORM_RMS, NORM_LAYER = range(3)
ROPE_NONE, ROPE_HALF, ROPE_INTERLEAVED = range(3)
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}

PLAIN = dict(op="attend", heads=32, kv_heads=32, dim=128, dtype="f16", page=64, seqs=1, len_min=1024,
             len_max=1024, new=1, ragged=False, window=0, layers=1, fan=1, spread=1.0, norm=NORM_NONE,
             rope=ROPE_NONE, rope_dims=0, rope_base=10000.0, rope_factor=1.0, fused=False)


def _case(name, **kw):
    return dict(PLAIN, name=name, **kw)


def listed():
    return [
        # one sequence in the middle of an answer, heads of the 4096-wide stacks
        _case("attend_one", len_min=1000, len_max=1000),
        # eight sequences, ragged
        _case("attend_eight", seqs=8, len_min=200, len_max=8000, ragged=True),
        # one key-value head under 71 query heads (4544 = 71 x 64)
        _case("attend_one_kv_head", heads=71, kv_heads=1, dim=64, seqs=8, len_min=1500, len_max=32000),
        # speculative decoding, heads of the 2560-wide stack: five tokens at once
        _case("attend_speculative", dim=80, seqs=8, len_min=100, len_max=2040, new=5, ragged=True, page=16),
        # one long document, grouped heads
        _case("attend_long", kv_heads=8, len_min=131001, len_max=131001, dtype="bf16", page=128),
        # the largest: a full batch, heads of the 7168-wide stack
        _case("attend_batch", heads=56, kv_heads=56, seqs=64, len_min=300, len_max=4000, page=32),
        # eight sequences' next tokens: layer norm per head, half of each head rotated
        _case("append_decode", op="append", heads=64, kv_heads=64, dim=64, seqs=8, len_min=50, len_max=2000,
              norm=NORM_LAYER, rope=ROPE_HALF, rope_dims=32, rope_base=25000.0, fused=True),
        # pieces of long documents: grouped heads, far positions at scaled frequencies
        _case("append_chunk", op="append", kv_heads=8, seqs=16, new=64, len_min=300, len_max=4000,
              dtype="bf16", norm=NORM_RMS, rope=ROPE_INTERLEAVED, rope_dims=128, rope_factor=8.0, fused=True),
        # two candidates of one sequence in a small stack
        _case("grow_two", op="grow", heads=4, kv_heads=4, dim=64, layers=2, seqs=1, fan=2, len_min=37, len_max=37, page=16),
        # eight sequences, four candidates each, every layer of a 4096-wide stack
        _case("grow_beams", op="grow", layers=32, seqs=8, fan=4, len_min=20, len_max=90, page=16, new=2),
        # a small cache with many short sequences
        _case("compact_short", op="compact", kv_heads=8, seqs=64, len_min=10, len_max=300, page=16, spread=3.0),
        # several layers of a cache whose pool is to be cut to half
        _case("compact_layers", op="compact", kv_heads=8, layers=16, seqs=12, len_min=400, len_max=4000, page=64,
              spread=2.0, dtype="bf16"),
    ]


def draw(rng):
    """Another case of the same ranges: every head dimension and page size, all ways to share key-value
    heads, odd numbers of sequences and tokens."""
    def spread(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    largest = {c["op"]: 0 for c in listed()}
    for c in listed():
        largest[c["op"]] = max(largest[c["op"]], work(c)["bytes"])
    op = rng.choice(["attend", "attend", "attend", "append", "append", "grow", "compact"])
    while True:
        dim, dtype = rng.choice([64, 80, 96, 128, 128, 256]), rng.choice(["f16", "f16", "bf16"])
        kv = rng.choice([1, 2, 4, 8, 12, 32, 40])
        group = rng.choice([1, 1, 2, 3, 4, 8]) if kv > 1 else rng.choice([1, 7, 16, 32, 71])
        c = dict(PLAIN, op=op, heads=kv * group, kv_heads=kv, dim=dim, dtype=dtype,
                 page=rng.choice([8, 16, 32, 64, 128, 256]), seqs=spread(1, 64), len_max=spread(1, 60000),
                 ragged=rng.random() < 0.5)
        c["len_min"] = spread(1, c["len_max"])
        if op == "attend":
            c.update(new=rng.choice([1, 1, 1, 2, 3, 5, 8, spread(1, 64)]),
                     window=rng.choice([0, 0, 0, spread(16, 8192)]))
        elif op == "append":
            c.update(new=rng.choice([1, 1, 2, 5, spread(1, 64)]), norm=rng.choice([NORM_NONE, NORM_RMS, NORM_LAYER]),
                     rope=rng.choice([ROPE_NONE, ROPE_HALF, ROPE_INTERLEAVED]), rope_base=rng.choice([1e4, 25e3, 1e6]),
                     rope_factor=rng.choice([1.0, 1.0, 4.0, 32.0]), fused=rng.random() < 0.5)
            if c["rope"] != ROPE_NONE:
                c.update(rope_dims=rng.choice([dim, dim // 2, 16 * rng.randint(1, dim // 16)]))
        elif op == "grow":
            c.update(seqs=spread(1, 24), fan=rng.randint(1, 6), layers=spread(1, 32), len_max=spread(1, 400),
                     new=rng.choice([1, 1, 2, 8, 64]))
            c["len_min"] = spread(1, c["len_max"])
        else:
            c.update(layers=spread(1, 16), spread=round(rng.uniform(1.1, 4.0), 2), len_max=spread(1, 6000))
            c["len_min"] = spread(1, c["len_max"])
        if c["heads"] > 128 or c["heads"] * c["dim"] > 8192:
            continue
        if _n_pages(c) * c["layers"] * _page_values(c) * 2 > (5 << 30 if op == "attend" else 1 << 29):
            continue
        if work(c)["bytes"] <= largest[op] and work(c)["bytes"] >= 512:
            return c


# ---- sizes: functions of the case alone ------------------------------------------------------------


def _page_values(case):
    return 2 * case["kv_heads"] * case["page"] * case["dim"]


def _sequences(case):
    """(length with this step's tokens, tokens of this step) of every place."""
    rng = random.Random(1000 * case["seqs"] + case["len_max"])
    lens, news = [], []
    for b in range(case["seqs"]):
        n = case["new"]
        L = round(math.exp(rng.uniform(math.log(case["len_min"]), math.log(case["len_max"]))))
        if case["ragged"] and case["seqs"] > 1 and b:
            n = rng.randint(1, n)
            if rng.random() < 0.1:
                L = n = 0
        lens.append(max(L, n))
        news.append(n)
    return lens, news


def _pages_for(tokens, case):
    return -(-tokens // case["page"])


def _n_pages(case):
    lens, _ = _sequences(case)
    used = sum(_pages_for(n, case) for n in lens)
    if case["op"] == "compact":
        return max(used, round(used * case["spread"]))
    if case["op"] == "grow":
        return used + sum(case["fan"] * (_pages_for(n + case["new"], case) - n // case["page"]) for n in lens)
    return used + 3


def work(case):
    lens, news = _sequences(case)
    H, Hkv, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    row = 2 * D                                                       # bytes of a head's 16-bit row
    if case["op"] == "attend":
        window = case["window"] or 1 << 40
        keys = sum(min(L, window + n - 1) for L, n in zip(lens, news) if n)
        pairs = sum(min(L - n + 1 + t, window) for L, n in zip(lens, news) for t in range(n))
        return {"bytes": keys * Hkv * 2 * row + 2 * sum(news) * H * row, "flops": 4 * pairs * H * D}
    if case["op"] == "append":
        return {"bytes": sum(news) * 2 * (H + 2 * Hkv) * row, "flops": sum(news) * (H + Hkv) * D * 10}
    if case["op"] == "grow":
        # copies: every holder of a shared, partly filled page but one
        copied = sum((case["fan"] - 1) * (L % P) for L in lens)
        entries = sum(case["fan"] * _pages_for(L + case["new"], case) for L in lens)
        return {"bytes": copied * case["layers"] * 4 * Hkv * row + 8 * entries, "flops": 0}
    used, total = sum(_pages_for(n, case) for n in lens), _n_pages(case)
    moved = used * (total - used) / total
    return {"bytes": moved * case["layers"] * 2 * 2 * _page_values(case) + 8 * used, "flops": 0}


# ---- what a program has in hand -----------------------------------------------------------------------


class State:
    pass


def rope_frequencies(case):
    """Radians per position of every rotated pair; `rope_factor` > 1 slows the low ones down for longer
    contexts (those with less than one turn in 8192 positions by the factor, those with more than 32 not
    at all, in between by a share of both)."""
    f = []
    for i in range(case["rope_dims"] // 2):
        w = case["rope_base"] ** (-2.0 * i / case["rope_dims"])
        turns = 8192 * w / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
        f.append(w * keep + w / case["rope_factor"] * (1.0 - keep))
    return f


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev, dt = "cuda", DTYPES[case["dtype"]]
    lens, news = _sequences(case)
    H, Hkv, D, P, n_pages = case["heads"], case["kv_heads"], case["dim"], case["page"], _n_pages(case)
    st = State()
    st.case, st.lens, st.news = case, lens, news
    st.pages = torch.empty(case["layers"], n_pages, 2, Hkv, P, D, dtype=dt, device=dev)
    for layer in st.pages:
        layer.normal_(generator=g)
    slots = case["seqs"] * case["fan"]
    width = max(1, max(_pages_for(n + (case["new"] if case["op"] == "grow" else 0), case) for n in lens))
    order = torch.randperm(n_pages, generator=g, device=dev).tolist()
    table = torch.full((slots, width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        k = _pages_for(n, case)
        table[b, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
        at += k
    st.table = table.to(dev)
    st.lens_dev = torch.tensor(lens + [0] * (slots - len(lens)), dtype=torch.int32, device=dev)
    st.n_new = torch.tensor(news + [0] * (slots - len(lens)), dtype=torch.int32, device=dev)
    T = case["new"]
    if case["op"] in ("attend", "append"):
        def rows(heads):
            return torch.randn(slots, T, heads, D, generator=g, device=dev).to(dt)
        st.out = torch.zeros(slots, T, H, D, dtype=dt, device=dev)
        if case["op"] == "append" and case["fused"]:                   # as a fused projection leaves them
            qkv = rows(H + 2 * Hkv)
            st.q, st.k, st.v = qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:]
        else:
            st.q = rows(H)
            if case["op"] == "append":
                st.k, st.v = rows(Hkv), rows(Hkv)
    st.norms = None
    if case["norm"] != NORM_NONE:
        def weight(mean):
            return (mean + 0.2 * torch.randn(D, generator=g, device=dev)).to(dt)
        st.norms = [weight(1.0), weight(0.0), weight(1.0), weight(0.0)]   # q weight, q bias, k weight, k bias
        if case["norm"] == NORM_RMS:
            st.norms[1] = st.norms[3] = None
    st.freq = rope_frequencies(case)
    st.freq_dev = torch.tensor(st.freq, dtype=torch.float64, device=dev)
    st.rope_scale = 0.1 * math.log(case["rope_factor"]) + 1.0
    if case["op"] == "grow":
        st.src = torch.arange(slots, dtype=torch.int32, device=dev) % case["seqs"]
        st.keep = st.lens_dev[:case["seqs"]].repeat(case["fan"])
        st.grow_by = torch.full((slots,), T, dtype=torch.int32, device=dev)
    if own:
        from paper_2312_11514_b200 import runtime
        st.kv = runtime.KvCache(
            n_layers=case["layers"], n_heads=H, n_kv_heads=Hkv, head_dim=D, dtype=dt, page_tokens=P, n_pages=n_pages,
            max_seqs=slots, max_pages=width, max_new=T, window=case["window"], norm=case["norm"], norm_eps=1e-5,
            rope=case["rope"], rope_dims=case["rope_dims"], rope_freq=st.freq, rope_scale=st.rope_scale,
            pages=st.pages)
        st.kv.load(st.lens_dev, st.table, st.n_new)
        st.state = {"pages": st.pages, "lens": st.kv.lens, "table": st.kv.table, "refs": st.kv.refs}
    else:
        st.now_lens, st.now_table = st.lens_dev.clone(), st.table.clone()
    return st


# ---- one pass -------------------------------------------------------------------------------------------


def run(state):
    op = state.case["op"]
    if own:
        kv = state.kv
        if op == "attend":
            return {"out": kv.attention(0, state.q, out=state.out)}
        if op == "append":
            q = kv.append(0, state.q, state.k, state.v, q_out=state.out, norms=state.norms)
            return {"q": q, "pages": state.pages}
        if op == "grow":
            kv.fork(state.src, state.keep)
            kv.reserve(state.grow_by)
        else:
            kv.load(state.lens_dev, state.table)
            kv.compact()
        return state.state
    return {"attend": _plain_attend, "append": _plain_append, "grow": _plain_grow, "compact": _plain_compact}[op](state)


def _plain_attend(st):
    c = st.case
    Hkv, D, P = c["kv_heads"], c["dim"], c["page"]
    G = c["heads"] // Hkv
    for b, (L, n) in enumerate(zip(st.lens, st.news)):
        if n == 0:
            continue
        first = max(0, L - n + 1 - c["window"]) if c["window"] else 0
        p0 = first // P
        held = st.pages[0][st.table[b, p0:_pages_for(L, c)].long()]    # [pages][2][Hkv][P][D]
        kv = held.permute(1, 2, 0, 3, 4).reshape(2, Hkv, -1, D)[:, :, :L - p0 * P].float()
        q = st.q[b, :n].float().reshape(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D)
        s = torch.matmul(q, kv[0].transpose(1, 2)) * (1.0 / math.sqrt(D))
        if n > 1 or c["window"]:
            at = torch.arange(p0 * P, L, device=s.device)
            upto = torch.arange(L - n, L, device=s.device).repeat_interleave(G)[:, None]
            hide = at[None, :] > upto
            if c["window"]:
                hide = hide | (at[None, :] <= upto - c["window"])
            s = s.masked_fill(hide[None], float("-inf"))
        p = torch.exp(s - s.amax(dim=2, keepdim=True))
        o = torch.matmul(p, kv[1]) / p.sum(dim=2, keepdim=True)
        st.out[b, :n] = o.reshape(Hkv, n, G, D).permute(1, 0, 2, 3).reshape(n, c["heads"], D).to(st.out.dtype)
    return {"out": st.out}


def _plain_norm(x, kind, w, b):
    if kind == NORM_RMS:
        return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-5) * w.float()
    if kind == NORM_LAYER:
        x = x - x.mean(dim=-1, keepdim=True)
        return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-5) * w.float() + b.float()
    return x


def _plain_rotate(x, pos, st):
    kind, R = st.case["rope"], st.case["rope_dims"]
    if kind == ROPE_NONE:
        return x
    a = pos.double()[..., None] * st.freq_dev                          # far positions: angles in 64 bits
    cos, sin = (st.rope_scale * torch.cos(a)).float()[:, :, None], (st.rope_scale * torch.sin(a)).float()[:, :, None]
    y = x.clone()
    u, v = (x[..., :R // 2], x[..., R // 2:R]) if kind == ROPE_HALF else (x[..., 0:R:2], x[..., 1:R:2])
    lo, hi = u * cos - v * sin, u * sin + v * cos
    if kind == ROPE_HALF:
        y[..., :R // 2], y[..., R // 2:R] = lo, hi
    else:
        y[..., 0:R:2], y[..., 1:R:2] = lo, hi
    return y


def _plain_append(st):
    c, dt, P = st.case, st.out.dtype, st.case["page"]
    t = torch.arange(c["new"], device="cuda")
    live = t[None] < st.n_new[:, None]
    pos = (st.lens_dev - st.n_new)[:, None] + t[None]
    n = st.norms or [None] * 4
    q = _plain_rotate(_plain_norm(st.q.float(), c["norm"], n[0], n[1]), pos, st).to(dt)
    k = _plain_rotate(_plain_norm(st.k.float(), c["norm"], n[2], n[3]), pos, st).to(dt)
    st.out[live] = q[live]
    b, _ = torch.nonzero(live, as_tuple=True)
    at = pos[live].long()
    page = st.table[b, at // P].long()
    st.pages[0][page, 0, :, at % P] = k[live]
    st.pages[0][page, 1, :, at % P] = st.v[live]
    return {"q": st.out, "pages": st.pages}


def _references(table, n_pages):
    held = table[table >= 0].long()
    refs = torch.zeros(n_pages, dtype=torch.int32, device=table.device)
    return refs.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))


def _plain_grow(st):
    P, n_pages = st.case["page"], st.pages.shape[1]
    lens, n = st.keep.long(), st.grow_by.long()
    slot = torch.arange(lens.numel(), device="cuda")
    j = torch.arange(st.now_table.shape[1], device="cuda")
    have = (lens + P - 1) // P
    table = torch.where(j[None] < have[:, None], st.now_table[st.src.long()], -1)
    refs = _references(table, n_pages)
    # a partly filled page that another place holds too is copied, unless all who hold it grow
    # now and this is the first of them
    last, rest = lens // P, lens % P
    tail = torch.where((n > 0) & (rest > 0), table.gather(1, last.clamp(max=j.numel() - 1)[:, None])[:, 0].long(), -1)
    at = tail.clamp(min=0)
    growers = torch.zeros(n_pages, dtype=torch.int64, device="cuda").index_add_(0, at, (tail >= 0).long())
    first = torch.full((n_pages,), lens.numel(), device="cuda").scatter_reduce_(
        0, at, torch.where(tail >= 0, slot, lens.numel()), "amin")
    copy = (tail >= 0) & (refs[at] > 1) & ~((growers[at] == refs[at]) & (first[at] == slot))
    more = (lens + n + P - 1) // P - have
    take = more + copy.long()
    begin = torch.cumsum(take, 0) - take
    free = torch.nonzero(refs == 0)[:, 0]
    c = torch.nonzero(copy)[:, 0]
    src, dst = tail[c], free[begin[c]]
    table[c, last[c]] = dst.to(table.dtype)
    new = torch.nonzero((j[None] >= have[:, None]) & (j[None] < (have + more)[:, None]))
    b, at = new[:, 0], new[:, 1]
    table[b, at] = free[begin[b] + copy.long()[b] + at - have[b]].to(table.dtype)
    keep = (torch.arange(P, device="cuda")[None] < rest[c][:, None])[:, None, None, :, None]
    for layer in st.pages:
        layer[dst] = torch.where(keep, layer[src], layer[dst])
    st.now_lens, st.now_table = (lens + n).to(torch.int32), table
    return {"pages": st.pages, "lens": st.now_lens, "table": table, "refs": _references(table, n_pages)}


def _plain_compact(st):
    n_pages = st.pages.shape[1]
    refs = _references(st.table, n_pages)
    used = refs > 0
    n_used = used.sum()
    page = torch.arange(n_pages, device="cuda")
    holes = torch.nonzero(~used & (page < n_used))[:, 0]
    movers = torch.nonzero(used & (page >= n_used))[:, 0].flip(0)
    to = page.clone()
    to[movers] = holes
    for layer in st.pages:
        layer[holes] = layer[movers]
    table = torch.where(st.table >= 0, to[st.table.clamp(min=0).long()].to(torch.int32), -1)
    return {"pages": st.pages, "lens": st.lens_dev, "table": table, "refs": _references(table, n_pages)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(st)
    if case["op"] == "append":
        return _exact_append(st)
    return _exact_pages(st)


def _exact_attend(st):
    """Head by head; the keys of a token are gathered one page entry per key."""
    c = st.case
    D, P, G = c["dim"], c["page"], c["heads"] // c["kv_heads"]
    tokens = sum(n for n in st.news)
    if tokens * c["kv_heads"] > 30000:
        return None
    out = torch.zeros(st.out.shape, dtype=torch.float64, device="cuda")
    for b in range(c["seqs"]):
        for t in range(st.news[b]):
            p = st.lens[b] - st.news[b] + t
            key = torch.arange(max(0, p + 1 - c["window"]) if c["window"] else 0, p + 1, device="cuda")
            page, row = st.table[b].long()[key // P], key % P
            for h in range(c["kv_heads"]):
                K = st.pages[0, page, 0, h, row].to(torch.float64)
                V = st.pages[0, page, 1, h, row].to(torch.float64)
                q = st.q[b, t, h * G:(h + 1) * G].to(torch.float64)
                w = torch.exp((q @ K.T / D ** 0.5) - (q @ K.T / D ** 0.5).amax(1, keepdim=True))
                out[b, t, h * G:(h + 1) * G] = (w @ V) / w.sum(1, keepdim=True)
    return {"out": out}


def _exact_append(st):
    """All tokens as complex numbers: a rotation is a product with exp(i angle)."""
    c, P = st.case, st.case["page"]
    if st.pages.numel() > 400_000_000:
        return None

    def normed(x, w, b):
        x = x.to(torch.float64)
        if c["norm"] == NORM_NONE:
            return x
        if c["norm"] == NORM_LAYER:
            x = x - x.mean(-1, keepdim=True)
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-5) * w.to(torch.float64)
        return x if b is None else x + b.to(torch.float64)

    def turned(x, p):                                                   # [n][heads][D] at position p
        R = c["rope_dims"]
        if c["rope"] == ROPE_NONE:
            return x
        turn = torch.polar(torch.full_like(st.freq_dev, st.rope_scale), p.double()[:, None] * st.freq_dev)[:, None]
        if c["rope"] == ROPE_HALF:
            z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous()) * turn
            return torch.cat([z.real, z.imag, x[..., R:]], dim=-1)
        z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous()) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., R:]], dim=-1)

    n = st.norms or [None] * 4
    q_out = torch.zeros(st.out.shape, dtype=torch.float64, device="cuda")
    pages = st.pages.to(torch.float64)
    for b in range(c["seqs"]):
        m = st.news[b]
        if not m:
            continue
        p = torch.arange(st.lens[b] - m, st.lens[b], device="cuda")
        q_out[b, :m] = turned(normed(st.q[b, :m], n[0], n[1]), p)
        k = turned(normed(st.k[b, :m], n[2], n[3]), p)
        for t in range(m):
            at = st.lens[b] - m + t
            page = int(st.table[b, at // P])
            pages[0, page, 0, :, at % P] = k[t]
            pages[0, page, 1, :, at % P] = st.v[b, t].to(torch.float64)
    return {"q": q_out, "pages": pages}


def _exact_pages(st):
    """The bookkeeping one entry at a time, in plain lists."""
    c, P, n_pages = st.case, st.case["page"], st.pages.shape[1]
    table = [[p for p in row if p >= 0] for row in st.table.tolist()]
    width, lens, copies = st.table.shape[1], st.lens_dev.tolist(), []
    if c["op"] == "compact":
        used = sorted({p for row in table for p in row})
        holes = sorted(set(range(len(used))) - set(used))
        to = dict(zip(reversed(used), holes))
        to = {s: d for s, d in to.items() if s >= len(used)}
        copies = [(s, d, P) for s, d in to.items()]
        table = [[to.get(p, p) for p in row] for row in table]
    else:
        n = c["new"]
        lens = [lens[b % c["seqs"]] for b in range(len(table))]
        table = [list(table[b % c["seqs"]][:-(-lens[b] // P)]) for b in range(len(table))]
        held = {}
        for b, row in enumerate(table):
            for p in row:
                held.setdefault(p, []).append(b)
        free = iter([p for p in range(n_pages) if p not in held])
        grown = []
        for b, row in enumerate(table):
            row = list(row)
            if n and lens[b] % P:
                p = row[lens[b] // P]
                ends_here = [o for o in held[p] if lens[o] // P < len(table[o]) and table[o][lens[o] // P] == p]
                if len(held[p]) > 1 and not (len(ends_here) == len(held[p]) and b == min(held[p])):
                    row[lens[b] // P] = next(free)
                    copies.append((p, row[lens[b] // P], lens[b] % P))
            while len(row) * P < lens[b] + n:
                row.append(next(free))
            grown.append(row)
        table, lens = grown, [x + n for x in lens]
    refs = [0] * n_pages
    for row in table:
        for p in row:
            refs[p] += 1
    pages = None
    if st.pages.numel() <= 400_000_000:
        pages = st.pages.to(torch.float64)
        for s, d, r in copies:
            pages[:, d, :, :, :r] = pages[:, s, :, :, :r]
    whole = [row + [-1] * (width - len(row)) for row in table]
    as_int = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    return {"pages": pages, "lens": as_int(lens), "table": as_int(whole), "refs": as_int(refs)}
