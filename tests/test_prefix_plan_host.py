"""How attention over shared prefixes plans a call, by the workspace that it asks for (CPU)."""

from paper_2504_03775_amd import flowkv as fk

ws = fk.flowkv_prefix_attention_workspace


def test_split_tokens_holds_where_there_is_nothing_to_share():
    """Records of a row: its tokens by split_tokens, as for chunk attention."""
    full = fk.flowkv_chunk_attention_workspace
    record = 130 * 4
    # 4 single tokens of 8 heads of 128 behind up to 600 in all: 10 splits of 64, 5 of 128
    for groups, prefix in ((0, 0), (1, 0)):
        assert ws(4, 4, 8, 2, 128, groups, 1, 4, 600, prefix, 64) == 4 * 8 * 10 * record
        assert ws(4, 4, 8, 2, 128, groups, 1, 4, 600, prefix, 128) == 4 * 8 * 5 * record
        for n, new, split in ((4, 1, 64), (700, 600, 64), (700, 600, 4096), (9, 3, 1024)):
            assert ws(n, 4, 8, 2, 128, groups, new, n, 5000, prefix, split) == \
                full(n, 4, 8, 2, 128, new, 5000, split)
    # no group: a prefix's tokens are as many more of the requests' own
    assert ws(4, 4, 8, 2, 128, 0, 1, 4, 200, 400, 64) == 4 * 8 * 10 * record
