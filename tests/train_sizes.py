"""Layer sizes (T, d, f, gated, dtype) that make the training path's products take every tile, with and without ranges of
the reduction, gated and un-gated, reductions of several rounds of the tile's ring among them, and rows that are aligned and
not.  test_plain_plan.py asks the choice whether that is still so; test_gpu_train_tiles.py runs them."""

SIZES = [(T, d, f, bool(gated), "f32") for T, d, f, gated in (
    (1, 8, 1, 0), (7420, 256, 1, 0), (1, 304, 8214, 0), (1, 296, 5504, 1), (466, 5864, 1, 1), (6878, 8, 134, 0), (5691, 8, 112, 1),
    (6466, 784, 65, 1), (1102, 1096, 1024, 0), (66, 4680, 2326, 1))]
SIZES += [(T, d, f, bool(gated), "bf16") for T, d, f, gated in (
    (2, 584, 592, 0), (1, 592, 10854, 1), (5455, 3104, 1, 0), (1, 4280, 6273, 0), (8703, 8, 194, 1), (5858, 3176, 1, 1),
    (578, 5024, 8, 1), (790, 8, 9736, 0), (1, 3384, 9499, 1), (7816, 3168, 2, 1), (2712, 8, 8496, 0), (5928, 4240, 8, 0),
    (33, 4432, 1882, 0), (112, 264, 11294, 0), (5917, 8, 4309, 1), (8467, 456, 131, 0), (274, 160, 11688, 0), (295, 144, 10946, 1),
    (142, 432, 8896, 1), (833, 5232, 130, 1), (5675, 136, 11332, 0), (278, 6112, 5584, 1), (385, 5792, 8934, 0), (8749, 440, 5848, 1))]
