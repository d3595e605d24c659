"""Sizes of the experts' products (m rows, experts, n, k) that between them launch every kernel, for aligned operands and others: the host
test holds the list to what the library launches, so the GPU tests that run these sizes keep reaching what they are for."""
SIZES = [
    (8192, 16, 5632, 2048), (16384, 32, 5632, 2048), (8, 64, 2816, 1024), (777, 7, 1000, 682), (777, 7, 1000, 684), (300, 8, 2048, 2048), (4000, 1, 256, 512),
    (4096, 64, 1024, 128), (3000, 5, 1024, 512), (9000, 3, 300, 2000), (1, 1, 1, 1), (64, 8, 512, 512), (14769, 1, 307, 501), (12000, 12, 2914, 3368),
    (2000, 100, 3215, 1333), (600, 2, 4096, 1024), (6017, 1, 894, 5695), (18576, 35, 2, 19), (135, 6, 222, 1198), (283, 2, 1335, 6320),
]
