"""Plain restatement of the paged key-value cache for the tests: tables as Python lists, attention and
rotation in 64 bits, and the error bounds that the kernels' arithmetic implies."""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # half a step, relative


class Tables:
    """What the calls of lif_kv.h say about lengths, tables and free pages, one entry at a time."""

    def __init__(self, max_seqs, max_pages, n_pages, page, max_new):
        self.P, self.n_pages, self.max_pages, self.max_new = page, n_pages, max_pages, max_new
        self.lens, self.n_new = [0] * max_seqs, [0] * max_seqs
        self.rows = [[] for _ in range(max_seqs)]

    def refs(self):
        r = [0] * self.n_pages
        for row in self.rows:
            for p in row:
                r[p] += 1
        return r

    def free(self):
        return [p for p, r in enumerate(self.refs()) if r == 0]

    def _pages(self, n):
        return -(-n // self.P)

    def reserve(self, n_new):
        """Returns (status name or None, [(source, destination, rows)])."""
        if any(n < 0 or n > self.max_new for n in n_new):
            self.n_new = [0] * len(n_new)
            return "invalid", []
        refs, free = self.refs(), iter(self.free())
        rows, copies, taken = [list(r) for r in self.rows], [], 0
        full = False
        for b, n in enumerate(n_new):
            if n and self.lens[b] % self.P:
                p = self.rows[b][-1]
                leavers = [o for o, m in enumerate(n_new) if m and self.lens[o] % self.P and self.rows[o][-1] == p]
                if refs[p] > 1 and not (len(leavers) == refs[p] and min(leavers) == b):
                    d = next(free, None)
                    full = full or d is None
                    rows[b][-1] = d
                    copies.append((p, d, self.lens[b] % self.P))
            while len(rows[b]) < self._pages(self.lens[b] + n):
                d = next(free, None)
                full = full or d is None
                rows[b].append(d)
            full = full or len(rows[b]) > self.max_pages
        if full:
            self.n_new = [0] * len(n_new)
            return "capacity", []
        self.rows, self.n_new = rows, list(n_new)
        self.lens = [a + n for a, n in zip(self.lens, n_new)]
        return None, copies

    def fork(self, src=None, length=None):
        src = list(range(len(self.lens))) if src is None else src
        length = [-1] * len(src) if length is None else length
        for s, n in zip(src, length):
            if s < -1 or s >= len(src) or (s >= 0 and not -1 <= n <= self.lens[s]):
                return "invalid"
        lens = [0 if s < 0 else self.lens[s] if n == -1 else n for s, n in zip(src, length)]
        self.rows = [[] if s < 0 else self.rows[s][:self._pages(n)] for s, n in zip(src, lens)]
        self.lens, self.n_new = lens, [0] * len(src)
        return None

    def load(self, lens, rows, n_new):
        self.lens, self.n_new, self.rows = list(lens), list(n_new), [list(r) for r in rows]

    def compact(self):
        used = [p for p, r in enumerate(self.refs()) if r]
        holes = [p for p in self.free() if p < len(used)]
        to = dict(zip(reversed(used), holes))
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        return [(s, d, self.P) for s, d in to.items()]

    def check(self, kv):
        torch.cuda.synchronize()
        assert kv.lens.tolist() == self.lens
        assert kv.n_new.tolist() == self.n_new
        want = [row + [-1] * (self.max_pages - len(row)) for row in self.rows]
        assert kv.table.tolist() == want
        assert kv.refs.tolist() == self.refs()
        assert kv.stats()["free"] == len(self.free())


def held(pages, layer, row, n, what):
    """Tokens 0 .. n-1 of a sequence: [n_kv_heads][n][D] in 64 bits."""
    if n == 0:
        return pages.new_zeros(pages.shape[3], 0, pages.shape[5], dtype=torch.float64)
    x = pages[layer, torch.tensor(row, device=pages.device), what]          # [pages][heads][P][D]
    return x.permute(1, 0, 2, 3).reshape(pages.shape[3], -1, pages.shape[5])[:, :n].double()


def attention(q, pages, layer, row, tokens, news, window=0, scale=None):
    """Reference of one sequence: q [news][H][D]; returns out [news][H][D] in 64 bits and the bound on a
    kernel's error, element by element.

    The kernel: scores are fp32 sums of D exact products, each addition off by at most 2^-23 (chopped)
    of the sum of magnitudes; so a weight is off by a factor exp(ds), ds = (D + 8) 2^-23 scale sum|q k|
    plus 2^-21 for the exponential and its argument's rounding (|argument| <= 2^6 at weights that
    matter: 2^-24 2^6 = 2^-18, so 2^-17 in all).  It is then rounded to 16 bits: off by the half step u
    relative, and in fp16 by at most 2^-25 absolute below 2^-14 (the largest weight is 1).  With A =
    sum w |v| / sum w the quotient moves by (relative error of a weight) * (A + |out|); the fp32 sums over
    L keys by (L + 64) 2^-23 of the same; and the output is rounded once: u |out| (fp16: 2^-25 at least)."""
    H, D = q.shape[1], q.shape[2]
    K, V = held(pages, layer, row, tokens, 0), held(pages, layer, row, tokens, 1)
    G = H // K.shape[0]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    u, sub = U[q.dtype], 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    out = torch.zeros(news, H, D, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    for t in range(news):
        p = tokens - news + t
        lo = max(0, p + 1 - window) if window else 0
        for h in range(K.shape[0]):
            x = q[t, h * G:(h + 1) * G].double()
            k, v = K[h, lo:p + 1], V[h, lo:p + 1]
            s = x @ k.T * scale
            w = torch.exp(s - s.amax(1, keepdim=True))
            w = w / w.sum(1, keepdim=True)
            o = w @ v
            ds = (D + 8) * 2.0 ** -23 * scale * (x.abs() @ k.abs().T).amax(1, keepdim=True) + 2.0 ** -17
            rel = u + ds + (p + 1 - lo + 64) * 2.0 ** -23
            A = w @ v.abs()
            out[t, h * G:(h + 1) * G] = o
            bound[t, h * G:(h + 1) * G] = u * o.abs() + rel * (1 + rel) * (A + o.abs()) + \
                sub * (1 + (p + 1 - lo) * 2 * v.abs().amax())
    return out, bound


def rotated(x, pos, norm, weight, bias, eps, rope, dims, freq, rope_scale):
    """Reference of append for one token: x [heads][D] -> (y, bound) in 64 bits.

    The kernel: mean and sum of squares over D elements in fp32 (D 2^-24 relative, halved by the root),
    a handful of roundings in the affine part; angles off by pi 2^-24 and their sines by 2 ulp (2^-23);
    so y is off by (D + 32) 2^-24 of the magnitudes that go into it, and rounded once."""
    u, D = U[x.dtype], x.shape[-1]
    c = (D + 32) * 2.0 ** -24
    y = x.double()
    mag = y.abs()
    if norm:
        if norm == 2:
            mean = y.mean(-1, keepdim=True)
            mag = mag + y.abs().mean(-1, keepdim=True)      # what the subtraction of the mean loses
            y = y - mean
        inv = 1.0 / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
        b = torch.zeros_like(weight).double() if bias is None else bias.double()
        y, mag = y * inv * weight.double() + b, mag * inv * weight.double().abs() + b.abs()
    if rope:
        a = pos * torch.tensor(freq, dtype=torch.float64, device=x.device)
        cos, sin = rope_scale * torch.cos(a), rope_scale * torch.sin(a)
        first = torch.arange(dims // 2, device=x.device) * (1 if rope == 1 else 2)
        second = first + (dims // 2 if rope == 1 else 1)
        p, q, mp, mq = y[:, first], y[:, second], mag[:, first], mag[:, second]
        y, mag = y.clone(), mag.clone()
        y[:, first], y[:, second] = p * cos - q * sin, p * sin + q * cos
        mag[:, first] = mag[:, second] = (mp + mq) * abs(rope_scale)
    exact = not norm and not rope
    floor = 2.0 ** -25 if x.dtype == torch.float16 else 0.0
    return y, torch.zeros_like(y) if exact else u * (y.abs() + c * mag) + c * mag + floor
