"""Products (m, n, k) that between them take every kernel of vsa2_fp8_matmul on a B200 (148 SMs), with sizes on a tile's edge and off it."""
SHAPES = [
    # tiles of 32 columns: one to 32 rows of A, B ragged; K in ranges, and not (few blocks, or tiles for all SMs)
    (1, 128, 128), (31, 1160, 129), (32, 200, 4100), (5, 19200, 1000),
    # tiles of 128 under a CTA alone (B has no rows for a second one); many tiles along A, in groups of 37 and a shorter one
    (33, 128, 130), (200, 72, 3000), (5200, 120, 130), (5204, 3, 2216),
    # pairs on tiles of 128: up to 128 rows of A, and where 224 columns waste more; K in ranges
    (128, 512, 128), (97, 136, 5000), (256, 4608, 640), (700, 904, 1100), (129, 256, 200), (1000, 264, 3000),
    # pairs on tiles of 224: ragged in A, in B, on the edge in both; K in ranges
    (300, 8192, 512), (4096, 4608, 640), (4093, 4616, 136), (1536, 640, 20000), (2978, 488, 17078),
    # many tiles along A: groups of 37 with a shorter last one of 16, one of one tile, whole groups alone; on tiles of 128 too
    (20000, 4608, 128), (8400, 2304, 100), (16576, 1024, 128), (8300, 2304, 100),
    # A's rows as lanes: ragged in B, in A, in both; groups of 37 along B with a shorter last one, one group, two whole ones
    (256, 9680, 512), (512, 15360, 640), (511, 15352, 640), (509, 6240, 648), (505, 6248, 1200), (250, 16576, 1000),
]
