"""Sizes (type, rows, in, out) of test_gpu_adapters_tiles: with them the tests run every kernel that the adapters'
plans can choose (test_adapter_plans checks that on the CPU)."""
SIZES = [
    ("bf16", 5, 40, 30),             # forward 64 x 64, gradient 64 x 128
    ("bf16", 50, 40, 31_003),        # 64 x 128, pass and split gradient
    ("bf16", 200, 70, 15_405),       # 64 x 128 of more than 64 rows
    ("bf16", 600, 53, 12_301),       # 128 x 128, split shrink
    ("bf16", 150, 45, 61_450),       # 256 x 256
    ("bf16", 70, 7_703, 8_301),      # gradient 128 x 128 split
    ("bf16", 70, 30_805, 2_101),     # gradient 128 x 128
    ("bf16", 300, 7_703, 8_301),     # gradient 256 x 256 split
    ("bf16", 520, 20_501, 2_101),    # gradient 256 x 256
    ("bf16", 40, 300, 4_205),        # gradient 64 x 128 split
    ("fp32", 5, 40, 65_541),         # forward 32 x 256
    ("fp32", 50, 40, 65_541),        # 64 x 256
    ("fp32", 600, 45, 6_607),        # 64 x 128, gradient 64 x 64 split
    ("fp32", 100, 300, 203),         # 64 x 64, gradient 128 x 128
    ("fp32", 100, 300, 2_003),       # gradient 128 x 128 split
    ("fp32", 20, 300, 203),          # gradient 32 x 256
    ("fp32", 20, 300, 2_003),        # gradient 32 x 256 split
    ("fp32", 50, 300, 203),          # gradient 64 x 256
    ("fp32", 50, 300, 2_003),        # gradient 64 x 256 split
    ("fp32", 50, 60, 101),           # gradient 64 x 64
]
