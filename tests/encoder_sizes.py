"""Sizes (rows, n_in, n_out) of the gated feed-forward that take every way its products are cut, for
16-bit types and for float: test_encoder_cuts.py checks that they do, test_gpu_encoder_tiles.py runs them."""

FFN_CUTS = [(3900, 72, 2000), (70, 2100, 200), (300, 264, 200), (20, 21, 17442), (132, 6863, 78), (735, 23, 20), (22, 20, 382),
            (726, 24, 339), (639, 7627, 292), (1390, 6084, 389), (16846, 259, 24), (7020, 1036, 423), (1289, 2668, 1028), (3665, 769, 1028),
            (12808, 20, 20), (77, 23, 20), (12888, 27, 135)]
