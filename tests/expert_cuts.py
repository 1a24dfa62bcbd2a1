"""More sizes of the experts' products: few rows split in two beside their
neighbours that are not, and 256 x 256 tiles of more experts than a wave has
lanes.  (tests/block_cuts.py has one size for every way they are cut.)"""
# operation (0 forward, 1 input gradient), type, rows, experts, d_in, d_out, splits of k: 32 x 128 tiles, of which the time
# model alone splits none; both sides of 128 tiles and of 2560 bytes of k
FEW = [
    (0, "bf16", 16, 16, 1280, 600, 2), (0, "bf16", 16, 16, 1279, 600, 1), (0, "bf16", 16, 40, 1301, 600, 2),
    (0, "bf16", 16, 17, 1280, 1024, 2), (0, "bf16", 17, 17, 1280, 1024, 1), (0, "bf16", 30, 40, 2048, 300, 2),
    (0, "f32", 30, 40, 640, 300, 2), (0, "f32", 30, 40, 639, 300, 1),
    (1, "bf16", 16, 16, 600, 1280, 2), (1, "bf16", 16, 16, 600, 1279, 1), (1, "bf16", 16, 40, 601, 1301, 2),
    (1, "f32", 30, 40, 300, 640, 2), (1, "f32", 30, 40, 300, 639, 1),
]
# as above, all of them in 256 x 256 tiles
BIG = [
    (0, "bf16", 18618, 70, 1000, 257), (1, "bf16", 18618, 70, 257, 1000), (0, "bf16", 23272, 130, 1000, 700),
    (1, "bf16", 23272, 130, 700, 1000), (0, "f32", 56815, 64, 1000, 700),
]
# weight gradients into padded rows: type, rows, experts, d_in, d_out, tile, whether k is split
PADDED = [
    ("f32", 5000, 3, 65, 131, "128x128", True), ("bf16", 1003, 1, 45, 54, "128x128", True),
    ("bf16", 2400, 2, 64, 64, "128x128", True), ("bf16", 1, 17, 247, 249, "128x128", False),
    ("f32", 1531, 5, 769, 1030, "64x128", False), ("bf16", 3783, 17, 2285, 2259, "256x256", False),
]
