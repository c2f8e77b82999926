"""Tables of layers that reach each way of sharing out a weight gradient's tiles: side 256 or 128, whole tiles alone, tiles
whose tokens are split, and both.  (tokens, rows, cols, gap) a layer; tests/test_grad_plan_tiles_cpu.py holds the library to
the side and shares named here, tests/test_gpu_weight_grad_tiles.py to the values."""

# name: (dtype, side, whole tiles, split tiles, layers)
CASES = {
    "whole_256": ("bf16", 256, True, False, [(300, 3001, 2900, 3)]),
    "whole_256_in_place": ("bf16", 256, True, False, [(700, 3001, 2900, 7)]),
    "split_256": ("bf16", 256, False, True, [(9001, 1800, 1790, 8)]),
    "split_256_odd": ("bf16", 256, False, True, [(12000, 1500, 1540, 3)]),
    "both_256": ("bf16", 256, True, True, [(1000, 4090, 4100, 6)]),
    "both_256_odd": ("bf16", 256, True, True, [(1000, 2300, 8180, 1)]),
    "mixed_256": ("bf16", 256, True, True, [(33, 300, 300, 5), (1100, 4090, 4100, 6), (0, 100, 50, 0), (700, 600, 700, 0)]),
    "both_128": ("bf16", 128, True, True, [(4100, 3001, 2900, 7)]),
    "mixed_128": ("bf16", 128, True, True, [(700, 600, 700, 0), (5000, 3001, 2900, 6), (33, 300, 300, 5)]),
    "whole_256_f32": ("f32", 256, True, False, [(65, 3001, 2900, 3)]),
    "split_256_f32": ("f32", 256, False, True, [(4100, 1500, 1540, 3)]),
    "both_256_f32": ("f32", 256, True, True, [(700, 4090, 4100, 0)]),
    "mixed_256_f32": ("f32", 256, True, True, [(33, 300, 300, 5), (500, 4090, 4100, 6), (0, 100, 50, 0), (300, 600, 700, 0)]),
    "both_128_f32": ("f32", 128, True, True, [(1000, 3001, 2900, 3)]),
}
