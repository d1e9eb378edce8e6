"""Sizes (rows, n_in, n_out) of the projections that take every way their products are cut, for 16-bit types and for
float: test_encoder_block_host.py checks that they do, test_gpu_linear.py runs them."""

LINEAR_CUTS = [(65, 33, 17), (300, 1024, 100), (100, 4000, 130), (257, 520, 1100), (1000, 72, 5000), (4096, 40, 4096), (130, 64, 192),
               (9000, 100, 1200), (8192, 2048, 2048), (2500, 2000, 2500), (12888, 27, 135), (600, 2048, 1030), (16384, 96, 24),
               (20, 21, 17442), (5000, 3000, 64), (70, 3500, 4096), (16384, 1100, 512), (300, 2100, 8200), (77, 3000, 20000),
               (40, 20, 30), (100, 4500, 130), (2816, 2048, 2816)]
