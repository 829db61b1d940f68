"""Sizes (tokens, width, vocabulary) that send the output head through each kernel that its plan can
choose: what the device tests run, and what the host check of the plan counts."""

# The three tiles, split and unsplit sums of one, two, three and more stages of 64, gradients in one
# and in two numbers, the few-token kernel with either number of rows and one, four, eight and sixteen
# waves to a group of them. Few are multiples of a vector or a tile.
SIZES = [
    (2, 1, 2), (494, 1, 2), (66, 72, 100), (159, 147, 157), (1943, 1, 3219), (3070, 8, 8565),
    (212, 251, 27634), (2645, 224, 3446), (5693, 104, 1568), (4796, 3359, 332), (460, 3018, 6814),
    (10, 1, 944), (333, 127, 86), (1, 1332, 4763), (1, 4200, 3135), (1957, 76, 3294),
    (103, 1197, 20836), (184, 3584, 5424), (970, 4342, 1661), (11, 2297, 2), (9, 1551, 5),
    (1875, 4518, 1), (3841, 1586, 2), (5069, 1419, 67), (88, 1728, 3484), (3386, 4424, 66),
    (68, 3808, 16042), (278, 4005, 10569), (6388, 760, 4068), (5077, 784, 7845),
    (4, 1024, 9001), (3, 8, 1_100_000), (8, 8192, 777), (4, 2048, 5001),
    (1, 768, 66_003), (2, 8, 70_001), (1, 513, 40_001), (16, 301, 60_007), (8, 65, 20_003),
    (9, 1001, 17_011), (3, 1281, 14_003)
]
