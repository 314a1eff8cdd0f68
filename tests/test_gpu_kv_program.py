"""A token's run of append, attention and FFN layer-step, layer by layer, each against its own reference."""
import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R
from paper_2312_11514_b200 import workloads as W

import kv_util as K
import parity_util as P
from test_gpu_kv import DEV, check_attention, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,norm,rope", [(4, 4, B.NORM_NONE, B.ROPE_HALF), (4, 1, B.NORM_RMS, B.ROPE_INTERLEAVED)])
def test_every_layer_of_every_token_as_the_formulas_have_it(heads, kv_heads, norm, rope):
    """Two sequences of two layers over a dozen tokens, drafts dropped and a sequence copied on the way: the appended
    queries, keys and values, the attention over the cache as it stands, and the layer-step's output and lists by the oracle."""
    cfg = W.CONFIGS["tiny"].scaled(n_streams=2, mean_fire=0.1)
    S, D, n_layers, page = 2, 64, 2, 8
    freq, eps = R.rope_frequencies(32), 1e-5
    pairs = [P.make_layer_pair(cfg, l, capacity=cfg.d_ff) for l in range(n_layers)]
    kv = R.KvCache(n_layers=n_layers, n_heads=heads, n_kv_heads=kv_heads, head_dim=D, n_pages=24, max_seqs=S, page_tokens=page,
                   norm=norm, norm_eps=eps, rope=rope, rope_dims=32, rope_freq=freq)
    ref = K.Tables(S, kv.max_pages, 24, page, 1)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    wq = torch.randn(n_layers, heads * D, (heads + 2 * kv_heads) * D, generator=g, device=DEV).half() * 0.06
    wo = torch.randn(n_layers, heads * D, heads * D, generator=g, device=DEV).half() * 0.06
    weights = [(1 + 0.2 * torch.randn(D, generator=g, device=DEV)).half() for _ in range(2)]
    norms = [weights[0], None, weights[1], None] if norm else None
    xs = W.make_inputs(cfg, device=DEV)
    assert xs.shape[2] == heads * D
    y = torch.empty(S, heads * D, dtype=torch.float32, device=DEV)
    for t in range(12):
        kv.reserve(ints([1] * S))
        assert ref.reserve([1] * S)[0] is None
        h = xs[t].clone()
        for l, (layer, oracle) in enumerate(pairs):
            qkv = (h @ wq[l]).view(S, 1, heads + 2 * kv_heads, D)
            q, k, v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads], qkv[:, :, heads + kv_heads:]
            q_out = kv.append(l, q, k, v, norms=norms)
            out = kv.attention(l, q_out, out=torch.full_like(q_out, 7))
            for b in range(S):
                pos = ref.lens[b] - 1
                for x, got, w in ((q, q_out[b, 0], weights[0]), (k, kv.pages[l, ref.rows[b][pos // page], 0, :, pos % page], weights[1])):
                    want, bound = K.rotated(x[b, 0], pos, norm, w, None, eps, rope, 32, freq, 1.0)
                    assert ((got.double() - want).abs() <= bound).all()
                assert torch.equal(kv.pages[l, ref.rows[b][pos // page], 1, :, pos % page], v[b, 0])
            check_attention(kv, ref.rows, ref.lens, [1] * S, q_out, out, layer=l)
            h = h + out.view(S, heads * D) @ wo[l]
            B.lif_decode_step(layer.handle, h, y)
            P.check_decode_step(layer, oracle, h.cpu().numpy(), y)
            h = h + 0.1 * y.half()
        if t == 6:
            kv.fork(None, ints([4, -1]))
            ref.fork(None, [4, -1])
        if t == 8:
            kv.fork(ints([1, 1]))
            ref.fork([1, 1])
    ref.check(kv)
    assert kv.stats()["status"] == B.LIF_OK
    kv.close()
    for layer, _ in pairs:
        layer.close()
