"""Host-only: the largest tables that a description may have."""
import pytest

from paper_2312_11514_b200 import binding as B

SHAPE = dict(n_layers=1, head_dim=64, page_tokens=256, n_pages=1, max_seqs=1)


def _tiles(d):
    rows = d["n_heads"] // d["n_kv_heads"] * d.get("max_new", 1)
    per_block = 16 if rows <= 16 else 128                    # heads of 64 elements
    return d["max_seqs"] * d["n_kv_heads"] * -(-rows // per_block) * d["max_pages"] * d["page_tokens"] // 64


@pytest.mark.parametrize("heads,kv_heads,max_new,max_seqs,max_pages,taken", [
    (128, 128, 1, 1, (1 << 22) - 1, False),                  # 2^31 - 512 tiles
    (126, 126, 1, 1, 1 << 22, False),
    (124, 124, 1, 1, 1 << 22, True),                         # 2^31 - 2^26
    (124, 124, 1, 1000, 4194, True),
    (125, 125, 1, 1, 4160749, True),
    (125, 125, 1, 1, 4160750, False),
    (71, 1, 64, 1000, 14000, True),                          # 36 blocks of rows
    (71, 1, 64, 1000, 14500, False)])
def test_tile_numbers_and_a_share_more_stay_in_32_bits(heads, kv_heads, max_new, max_seqs, max_pages, taken):
    """The plan of a step adds a share of the tiles (a 32nd of them at most) to a tile's number."""
    d = dict(SHAPE, n_heads=heads, n_kv_heads=kv_heads, max_new=max_new, max_seqs=max_seqs, max_pages=max_pages)
    tiles = _tiles(d)
    assert taken == (tiles <= 2 ** 31 - 2 ** 26)
    if taken:
        assert tiles + -(-tiles // 32) < 2 ** 31
        assert B.lif_kv_workspace_bytes(B.make_kv_desc(**d)) > 0
    else:
        with pytest.raises(B.LifError) as e:
            B.lif_kv_workspace_bytes(B.make_kv_desc(**d))
        assert e.value.code == B.LIF_ERR_INVALID_ARG
