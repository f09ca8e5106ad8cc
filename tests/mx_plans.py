"""Sizes of products with one matrix, (m, k, n), and what wc_linear_mx runs for them: the tile's kernel,
the parts of k, and whether the matrix's scales are copied.  Each kernel, with one part and with
more; test_mx_plans checks that the library takes these, test_gpu_mx_plans runs them."""

PLANS = [
    ((226, 115, 1326), "tile64 1 0"), ((750, 66, 716), "tile64 1 1"), ((348, 7107, 727), "tile64 2 1"),
    ((78, 4060, 109), "tile64 4 1"), ((65, 8185, 68), "tile64 8 0"), ((43, 8013, 102), "tile64 8 1"),
    ((147, 105, 18745), "tile128 1 0"), ((1817, 65, 2190), "tile128 1 1"), ((4299, 25907, 652), "tile128 2 1"),
    ((706, 12842, 1360), "tile128 4 1"), ((628, 25625, 770), "tile128 8 1"),
    ((251, 99, 8197), "tile128deep 1 0"), ((1331, 70, 1585), "tile128deep 1 1"),
    ((636, 8733, 1621), "tile128deep 2 1"), ((780, 13804, 660), "tile128deep 4 1"),
    ((391, 11737, 578), "tile128deep 8 1"),
    ((227, 113, 33441), "tile256 1 0"), ((3061, 64, 2997), "tile256 1 1"), ((1030, 2049, 8201), "tile256 1 1"),
    ((2100, 513, 4203), "tile256 1 1"), ((1482, 21363, 2716), "tile256 2 1"), ((1715, 23171, 1157), "tile256 4 1"),
    ((145, 35948, 5599), "tile256 8 0"), ((1102, 42183, 969), "tile256 8 1"),
    ((21, 64, 67), "slim 1 0"), ((100, 512, 512), "slim 1 0"),
    ((16, 4096, 300), "stream16 1 0"), ((9, 8193, 5000), "stream32 1 0"), ((13, 8192, 17000), "stream64 1 0")]
