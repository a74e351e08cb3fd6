"""Sizes that reach each way that attention over pages is computed, for tests that hold all of them to the same behaviour."""

PAGE = 16
# name: heads, clusters, bound of the rows' lengths, the rows, kernels that the call launches
SHORT, LONG = 592, 5008
ROWS = [560, 90, 577]
PATHS = {
    "rows by eight waves, clusters": (6, 2, SHORT, ROWS, ["paged_rows"]),
    "rows by eight waves, dense": (6, 6, SHORT, ROWS, ["paged_rows"]),
    "rows by four waves, clusters": (72, 9, SHORT, ROWS, ["paged_rows"]),
    "rows by four waves, dense": (72, 72, SHORT, ROWS, ["paged_rows"]),
    "rows in order, clusters": (72, 9, SHORT, ROWS + [301], ["paged_rows"]),
    "shares, clusters": (6, 2, LONG, ROWS, ["paged_scores", "paged_values", "paged_join"]),
    "shares, dense": (6, 6, LONG, ROWS, ["paged_attend", "paged_join"]),
    "shares of many heads, clusters": (180, 20, LONG, ROWS, ["paged_scores", "paged_values", "paged_join"]),
    "shares of many heads, dense": (180, 180, LONG, ROWS, ["paged_attend", "paged_join"]),
}
CACHES = ["f32", "bf16", "e4m3"]

# heads, clusters: batches of more rows than lanes, one of them long (their lengths are added up in two levels)
MANY_ROWS, LONGEST = [65, 130, 200, 300], 4200
MANY_HEADS = [(3, 2), (3, 3)]


def many_lengths(B):
    """Rows without a position at either end, inside and over a lane's whole share of the rows, a long one behind them."""
    lengths = [(37 * i + 11) % 90 for i in range(B)]
    for i in [0, 1, 2, *range(B // 2, B // 2 + 9), B - 2, B - 1]:
        lengths[i] = 0
    lengths[B // 2 + 10] = LONGEST
    return lengths


# rows, heads, clusters, tokens of a call: rows moved by waves that are dealt units of more rows than lanes
MOVED = [(70, 60, 12, 61), (130, 40, 40, 33)]
