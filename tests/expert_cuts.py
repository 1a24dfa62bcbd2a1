"""More sizes of the experts' products: few rows split in two beside their
neighbours that are not.  (tests/block_cuts.py has one size for every way they
are cut.)"""
# operation (0 forward, 1 input gradient), type, rows, experts, d_in, d_out, splits of k: 32 x 128 tiles, of which the time
# model alone splits none; both sides of 128 tiles and of 2560 bytes of k
FEW = [
    (0, "bf16", 16, 16, 1280, 600, 2), (0, "bf16", 16, 16, 1279, 600, 1), (0, "bf16", 16, 40, 1301, 600, 2),
    (0, "bf16", 16, 17, 1280, 1024, 2), (0, "bf16", 17, 17, 1280, 1024, 1), (0, "bf16", 30, 40, 2048, 300, 2),
    (0, "f32", 30, 40, 640, 300, 2), (0, "f32", 30, 40, 639, 300, 1),
    (1, "bf16", 16, 16, 600, 1280, 2), (1, "bf16", 16, 16, 600, 1279, 1), (1, "bf16", 16, 40, 601, 1301, 2),
    (1, "f32", 30, 40, 300, 640, 2), (1, "f32", 30, 40, 300, 639, 1),
]
