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
