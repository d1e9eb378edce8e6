"""Sequences of heads of more than 128 widths (lengths, heads, heads of q and k, dk, dv) that are long enough to be cut into
segments: test_delta_wide_host.py checks that they are, test_gpu_delta_wide.py runs them."""

WIDE = [([1100], 1, 1, 150, 40), ([1500, 0, 2100], 2, 1, 136, 72), ([1024], 2, 2, 256, 24), ([2100], 1, 1, 256, 40)]
