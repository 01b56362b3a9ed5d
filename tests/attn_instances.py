"""Batches that between them take every instance of the attention kernels: rows a tile, size
class of the heads, size class of the pages, a workgroup a tile or tiles shared out."""

# page, heads, G, dim, new tokens, lengths
CASES = [(page, heads, G, dim, news, lens)
         for heads, G, dims, few, many in (
             # tiles of 16 rows
             (2, 2, (16, 64), ([3, 1], [130, 70]), ([2, 1], [2600, 70])),
             (2, 3, (96, 128), ([3, 1], [130, 70]), ([2, 1], [2600, 70])),
             (1, 4, (144, 192, 256), ([3, 1], [130, 70]), ([2, 1], [2600, 70])),
             # of 32
             (2, 1, (48, 64), ([30, 20], [300, 70]), ([40, 3], [2600, 70])),
             (1, 2, (80, 128), ([15, 9], [300, 70]), ([20, 2], [2600, 70])),
             # of 128
             (1, 2, (32, 64), ([70, 9], [200, 9]), ([80, 3], [2600, 70])),
             (1, 3, (80, 112, 128), ([70, 9], [200, 9]), ([60, 3], [2600, 70])),
             (1, 2, (160, 208, 256), ([70, 9], [200, 9]), ([80, 3], [2600, 70])),
         )
         for news, lens in (few, many)
         for k, dim in enumerate(dims)
         for page in ((16, 64), (32, 128), (16, 128))[k]]

# causal, window: a window that leaves long tiles long, and a short one
MASKS = [(True, 0), (False, 0), (True, 1700), (False, 40), (True, 40)]
