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


def records(n_tokens, *rest):
    """Records a row of a shared call, by the workspace; None: not one of a whole number of them
    (work by the lengths: pieces), 0: none."""
    bytes_ = ws(n_tokens, *rest)
    row = n_tokens * rest[1] * (rest[3] + 2) * 4
    return bytes_ // row if bytes_ % row == 0 else None


def test_a_long_request_does_not_end_sharing_for_the_others():
    """63 single tokens beside one request of more, behind one prefix (32 heads of 128 on 8, 8
    of 128 on 1, 8 of 64 on 4): records of a prefix's splits and of the tokens behind it."""
    for hq, hk, d in ((32, 8, 128), (8, 1, 128), (8, 4, 64)):
        for prefix in (4000, 13000):
            for new in (1, 16, 17, 64, 100, 300, 512):
                n = 63 + new
                assert (records(n, 64, hq, hk, d, 1, new, n, 400, prefix) or 0) >= 2, (hq, new)
    # where the requests bring many rows on average, whole tiles read a prefix once for many
    for n, req, new in ((16 * 300, 16, 300), (64 * 17, 64, 17), (64 * 20, 64, 40), (15 + 2000, 16, 2000)):
        assert ws(n, req, 32, 8, 128, 1, new, n, 400, 4000) == \
            ws(n, req, 32, 8, 128, 0, new, n, 400, 4000), (n, req)
    # little saved: one prefix for one request, and for two requests of short ones
    for n, req, prefix in ((100, 1, 9000), (2, 2, 300)):
        assert ws(n, req, 32, 8, 128, 1, n // req, n, 400, prefix) == \
            ws(n, req, 32, 8, 128, 0, n // req, n, 400, prefix)
    # padding rows are nobody's: single tokens in a batch of 8,192 rows, as a captured call has them
    assert records(8192, 64, 32, 8, 128, 1, 1, 64, 400, 4000) >= 2


def test_the_rule_takes_no_plan_that_a_launch_cannot_hold():
    """100,000 requests, one of 100 new tokens and 50,000 tokens of its own: a workgroup for every
    split of every request's own would pass the lanes of a launch; whole tiles do not."""
    n, req = 100_099, 100_000
    assert ws(n, req, 32, 8, 128, 1, 100, n, 50_000, 13_000) == \
        ws(n, req, 32, 8, 128, 0, 100, 0, 63_000, 0)
    # where they fit
    for n, own in ((20_000, 60_000), (60_000, 30_000), (100_000, 20_000)):
        assert records(n, n, 32, 8, 128, 1, 1, n, own, 13_000) >= 2
