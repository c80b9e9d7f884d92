"""Further sizes (M, N, K) of the encoder's products: with those of encoder_shapes.py and the small ones of test_gpu_encoder.py every
variant that a call can launch is tested; test_encoder_routes.py holds them to it, type by type, linear and gated."""

MORE = [(2056, 978, 7376), (5019, 713, 327), (692, 5379, 3593), (429, 195, 6443), (5836, 689, 6375), (288, 8, 8), (813, 8, 2838),
        (204, 773, 1440)]

# few rows of many columns
FEW = [(1, 4669, 9), (1, 4081, 500), (8, 8195, 264), (16, 4099, 2048)]
