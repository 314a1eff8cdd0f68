"""Host-only checks of the paged key-value cache: descriptions, refused arguments, frequencies."""
import ctypes as C
import math

import pytest
import torch

from paper_2312_11514_b200 import binding as B
from paper_2312_11514_b200 import runtime as R

SHAPE = dict(n_layers=2, n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=32, max_seqs=4, max_pages=8)


def _bytes(**kw):
    return B.lif_kv_workspace_bytes(B.make_kv_desc(**dict(SHAPE, **kw)))


def test_workspace_grows_with_what_it_holds():
    n = _bytes()
    assert n > 0 and n % 256 == 0
    assert _bytes(n_pages=1 << 16) > n and _bytes(max_pages=1 << 12) > n and _bytes(max_new=64) > n
    assert _bytes(rope=B.ROPE_HALF, rope_dims=64) > n
    assert _bytes(n_layers=1024) == n                       # the tables serve every layer


@pytest.mark.parametrize("bad", [
    dict(n_layers=0), dict(n_layers=1025), dict(n_heads=0), dict(n_heads=9), dict(n_heads=1026), dict(n_kv_heads=0),
    dict(n_kv_heads=-2), dict(head_dim=72), dict(head_dim=0), dict(head_dim=512), dict(dtype=2), dict(dtype=-1),
    dict(page_tokens=24), dict(page_tokens=4), dict(page_tokens=512), dict(n_pages=0), dict(n_pages=(1 << 24) + 1),
    dict(max_seqs=0), dict(max_seqs=1025), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(max_new=0),
    dict(max_new=65), dict(window=-1), dict(scale=-0.1), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(norm=3), dict(norm=-1), dict(norm=1, norm_eps=-1e-6), dict(norm=2, norm_eps=float("nan")), dict(rope=3),
    dict(rope=1, rope_dims=0), dict(rope=1, rope_dims=31), dict(rope=1, rope_dims=66), dict(rope=0, rope_dims=64),
    dict(rope=2, rope_dims=64, rope_scale=float("nan")),
    dict(max_seqs=1024, max_pages=1 << 22, page_tokens=256, n_heads=128, n_kv_heads=128),   # more tiles than 32 bits
])
def test_descriptions_refused(bad):
    with pytest.raises(B.LifError) as e:
        _bytes(**bad)
    assert e.value.code == B.LIF_ERR_INVALID_ARG


def test_create_checks_pointers_and_frequencies_on_the_host():
    def create(freq=None, **kw):
        d = B.make_kv_desc(**dict(SHAPE, **kw), rope_freq=freq)
        d.dev_pages, d.dev_workspace, d.workspace_bytes = 0x10000, 0x20000, 1 << 40
        return d

    def code(d):
        out = C.c_void_p(0)
        return B.lib().lif_kv_create(C.byref(d), C.byref(out))

    d = create()
    assert B.lib().lif_kv_create(C.byref(d), None) == B.LIF_ERR_INVALID_ARG
    d.dev_pages = None
    assert code(d) == B.LIF_ERR_INVALID_ARG
    d = create()
    d.dev_workspace = None
    assert code(d) == B.LIF_ERR_INVALID_ARG
    d = create()
    d.dev_pages = 0x10008
    assert code(d) == B.LIF_ERR_ALIGNMENT
    d = create()
    d.dev_workspace = 0x20010
    assert code(d) == B.LIF_ERR_ALIGNMENT
    d = create()
    d.workspace_bytes = 64
    assert code(d) == B.LIF_ERR_INVALID_ARG
    assert code(create(rope=1, rope_dims=8)) == B.LIF_ERR_INVALID_ARG             # no frequencies
    for f in (float("nan"), 6.3, -7.0, float("inf")):
        freq = (C.c_double * 4)(1.0, 0.1, f, 0.001)
        assert code(create(freq, rope=1, rope_dims=8)) == B.LIF_ERR_INVALID_ARG, f


def test_calls_refuse_null_handles():
    lib = B.lib()
    rows = C.byref(B.KvRows(0x1000, 64, 64))
    for got in (lib.lif_kv_destroy(None), lib.lif_kv_get_state(None, C.byref(B.KvState())), lib.lif_kv_reset(None, None),
                lib.lif_kv_reserve(None, 0x1000, None), lib.lif_kv_append(None, 0, rows, rows, rows, None, 0x1000, None),
                lib.lif_kv_attention(None, 0, 0x1000, 0x1000, None), lib.lif_kv_fork(None, None, None, None),
                lib.lif_kv_load(None, 0x1000, 0x1000, None, None), lib.lif_kv_compact(None, None),
                lib.lif_kv_get_stats(None, (C.c_int32 * B.KV_CNT_LEN)()), lib.lif_kv_clear_status(None, None),
                lib.lif_kv_workspace_bytes(None, C.byref(C.c_size_t(0))),
                lib.lif_kv_workspace_bytes(C.byref(B.make_kv_desc(**SHAPE)), None)):
        assert got == B.LIF_ERR_INVALID_ARG


def test_cache_needs_a_device():
    if torch.cuda.is_available():
        pytest.skip("has one")
    with pytest.raises(RuntimeError, match="no CPU path"):
        R.KvCache(n_layers=1, n_heads=4, n_kv_heads=4, head_dim=64, n_pages=4, max_seqs=1)


def test_rope_frequencies():
    plain = R.rope_frequencies(8, 10000.0)
    assert plain == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-12)
    assert R.rope_frequencies(8, scaling="linear", factor=4.0) == pytest.approx([f / 4 for f in plain])
    ntk = R.rope_frequencies(8, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and ntk[-1] == pytest.approx(plain[-1] / 4)             # highest stays, lowest / factor
    parts = R.rope_frequencies(8, scaling="by_parts", factor=4.0, context=2048)
    turns = [2048 * f / (2 * math.pi) for f in plain]                           # 326, 33, 3.3, 0.33
    assert parts[0] == plain[0] and parts[1] == plain[1] and parts[3] == pytest.approx(plain[3] / 4)
    share = (turns[2] - 1) / 31
    assert parts[2] == pytest.approx(plain[2] * share + plain[2] / 4 * (1 - share))
    for bad in (dict(dims=7), dict(dims=0), dict(dims=8, base=0.0), dict(dims=8, scaling="other"),
                dict(dims=8, scaling="by_parts", factor=2.0), dict(dims=8, scaling="linear", factor=0.5)):
        with pytest.raises(ValueError):
            R.rope_frequencies(**bad)
