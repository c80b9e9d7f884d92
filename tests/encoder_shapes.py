"""Sizes (M, N, K) at which the encoder's products take each of their routes; test_encoder_rules.py holds them to it."""

# ragged against both tile sizes on every side; K short, K a multiple of 16 but not of a stage, K a multiple of nothing
TILES = [(4104, 2056, 200), (4104, 2056, 1040), (4104, 2056, 1100), (2100, 2100, 1040), (260, 260, 4100), (700, 300, 4000),
         (600, 700, 2000), (200, 4104, 2056), (4104, 200, 2056), (300, 520, 1100), (90, 520, 4112)]

# 8 bits: long enough for the scaled matrix instruction, in large tiles
TILES_8_BITS = TILES + [(4104, 2056, 2064), (4104, 2056, 2100), (2100, 2100, 2080)]
