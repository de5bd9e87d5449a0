"""Calls of attention over the four-bit cache, chosen by the kernels that they take (test_more_operator_forms.py holds that) and run by test_gpu_cache4_forms.py.
(cached, new tokens, query heads, KV heads, head_dim, page size, window, sinks)"""
NONE = 2 ** 31 - 1

# chunks in equal shares: cut items whose rows see tiles of sinks and then tiles of the window; sinks inside a tile, of several tiles, behind the window; single tokens and empty sequences beside them
SHARED_CHUNKS = [([3000, 2500, 3100], [300, 300, 299], 16, 8, 64, 16, 2500, 70), ([3000, 2500, 3100], [300, 300, 299], 16, 8, 128, 64, 2500, 5), ([3000, 2900, 3100], [300, 280, 299], 16, 8, 128, 32, 1300, 200),
                 ([3000, 100, 0, 3500, 3111], [400, 1, 0, 400, 9], 28, 4, 64, 128, 2000, 64), ([3000, 2999], [400, 397], 28, 4, 128, 16, 1900, 3), ([2600, 2000, 3001], [300, 299, 301], 16, 8, 64, 16, NONE, 0),
                 ([3300, 20], [350, 300], 32, 8, 128, 16, NONE, 0)]

# few rows in equal shares, by the rows of their tiles (float32: 16 at most)
SHARED_ROWS = [(4, ([4500, 3000, 77], [1, 1, 1], 16, 4, 128, 16, 4300, 70)), (8, ([3600, 2222, 0, 3300], [2, 2, 1, 0], 32, 8, 128, 64, NONE, 0)), (8, ([3600, 2222, 3], [1, 1, 1], 28, 4, 128, 16, 2900, 70)),
               (8, ([4000, 3900], [2, 1], 8, 2, 64, 32, 3500, 5)), (16, ([3600, 2222, 40], [4, 3, 1], 16, 4, 128, 16, 2900, 33)), (16, ([4000, 3900], [5, 5], 6, 2, 64, 16, NONE, 0)),
               (32, ([3600, 2222, 40], [8, 7, 1], 16, 4, 128, 16, 2900, 33)), (32, ([4000, 3900], [16, 10], 8, 2, 64, 64, 3000, 70))]

# chunks in float32: whole items, and equal shares
WHOLE_FLOATS = [([1500], [1300], 16, 8, 128, 16, NONE, 0), ([1500, 1700], [900, 500], 16, 8, 64, 32, 1400, 70)]
SHARED_FLOATS = [([2600, 2000, 3001], [120, 99, 1], 16, 8, 128, 64, NONE, 0), ([2600, 2000, 3001], [120, 0, 117], 14, 2, 64, 16, 1800, 70)]
