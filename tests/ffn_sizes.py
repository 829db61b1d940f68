"""Sizes (tokens, width, inner) that send the block's products through each of their kernels: what
the device tests run, and what the host check of the plan counts."""

# The larger tiles, split and unsplit sums, of one, two, three and more stages of 64. (The 64-row
# tile has the small sizes of test_gpu_feed_forward.py.) Few are multiples of a vector or a tile.
TILES = [
    (8214, 668, 8), (7434, 864, 208), (4419, 1287, 66), (7174, 1034, 9), (4779, 1687, 196),
    (2117, 2826, 130), (3363, 2326, 65), (18, 259, 5881), (5453, 2355, 129), (1733, 282, 3636),
    (70, 6148, 260), (25, 7208, 263), (132, 6258, 258), (74, 7176, 273), (157, 7569, 258),
    (197, 7301, 269), (8290, 65, 651), (7030, 10, 387), (8260, 17, 710), (8374, 138, 643),
    (8268, 74, 331), (8274, 142, 321), (974, 1330, 3613), (899, 927, 6760), (5519, 2831, 387),
    (1667, 2484, 5654), (906, 1931, 6791),
]

# Up to sixteen tokens: either number of rows of a workgroup, four, eight and sixteen waves.
FEW = [(t, k, f) for t in (1, 7, 8, 9, 15, 16)
       for k, f in ((1100, 1030), (2055, 512), (512, 2055), (1100, 9001), (4096, 1001))]
