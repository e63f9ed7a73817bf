"""Sizes at the ends of their ranges, for the calls whose launches go by a count of tiles (CPU)."""

from paper_2504_03775_amd import flowkv as fk

MOST = 2**31 - 1


def test_tiles_of_the_most_requests_and_new_tokens():
    """The tiles that the batch's tokens can have bound the requests' own, however many: a count
    past 64 bits (2^31 requests of 2^30 tokens of 2,048 rows) is not a small one."""
    chunk = fk.flowkv_chunk_attention_workspace
    window = fk.flowkv_window_attention_workspace
    prefix = fk.flowkv_prefix_attention_workspace
    for d in (64, 128):
        shape = (1, MOST, 2048, 1, d)
        for new in (1 << 30, MOST, (1 << 30) + 12345):
            assert chunk(*shape, new, 100_000) == chunk(*shape, 1000, 100_000) == 0
            assert window(*shape, new, 100_000, 50_000, 4) == 0
            assert prefix(*shape, 0, new, 0, 100_000, 0) == 0
            assert prefix(1, 1, 2048, 1, d, MOST, 1, new, 100, 9000, 64) == \
                prefix(1, 1, 2048, 1, d, MOST, 1, 1000, 100, 9000, 64)
