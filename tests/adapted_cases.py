"""Sizes of the tests of projections with adapters: the kernel that each is there for, (rows, heads, slots, tokens, width)."""
CASES = {
    "rows": [(1, 4, 2, 1, 64), (8, 16, 8, 1, 512), (2, 16, 16, 4, 192)],
    "stream": [(3, 32, 4, 5, 1024), (16, 32, 8, 1, 1280), (1, 32, 8, 32, 1280), (1, 72, 16, 64, 4096), (2, 128, 128, 1, 1024), (64, 12, 12, 1, 4096)],
    "tile": [(5, 7, 3, 30, 256), (2, 8, 8, 333, 128), (40, 6, 2, 3, 320)],
    "large": [(2, 16, 16, 801, 192), (4, 16, 16, 1025, 128), (1, 3, 3, 16384, 64)],
}
RANKS = [8, 16, 24, 64, 128]
# calls that go another way than those without adapters: in parts of rows that can be listed, and small tiles of more tokens
PARTS = [(43, 32, 32, 2, 256), (35, 72, 72, 4, 128), (1030, 1, 1, 3, 64)]
MORE = [(14, 72, 72, 32, 1024)]
