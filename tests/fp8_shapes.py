"""Sizes of 8-bit products that reach every kernel: shape and threads, a split sum or not, results of 16 bits or of 32. That
they do is asserted on the CPU (tests/test_fp8_shapes.py), what they give on the GPU (tests/test_gpu_fp8_shapes.py)."""

NARROW, WIDE = ("bf16", "f16"), ("f32",)
EVERY = NARROW + WIDE

#: M, N, K and the types of the results
SIZES = [
    # up to 16 rows of A: eight waves and sixteen, one tile of B's rows to a workgroup and two; the blocks of K come to
    # several rounds of a wave's loads, with and without a rest
    (16, 4200, 1153, EVERY), (5, 4097, 4608, EVERY), (16, 300, 8200, EVERY), (7, 129, 2048, EVERY),
    (8, 8200, 8200, EVERY), (16, 8195, 4224, EVERY),
    # up to 32
    (32, 4090, 4232, EVERY), (19, 333, 640, EVERY),
    # tiles of 64 x 128
    (130, 257, 900, EVERY), (300, 130, 1024, EVERY), (77, 500, 2090, EVERY), (65, 1000, 4096, EVERY),
    # of 128 x 64
    (8291, 129, 261, EVERY), (5463, 257, 512, NARROW), (2312, 769, 512, WIDE), (838, 515, 1962, NARROW), (775, 515, 2048, NARROW),
    (812, 516, 1926, WIDE), (647, 401, 3584, WIDE),
    # of 128 x 128
    (2000, 3001, 300, NARROW), (2312, 1679, 512, NARROW), (2995, 2500, 300, WIDE), (1678, 2309, 512, WIDE),
    (1811, 1116, 5273, NARROW), (974, 2086, 5632, NARROW), (717, 2787, 5312, WIDE), (1574, 1285, 5632, WIDE),
    # of 256 x 256, more than one to a compute unit among them
    (1290, 8894, 301, NARROW), (2563, 3100, 512, NARROW), (4097, 4100, 520, NARROW), (517, 2317, 13081, NARROW),
    (1215, 3342, 4608, NARROW),
]
