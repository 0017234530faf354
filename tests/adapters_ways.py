"""Sizes of products with adapters by the way that they take (csrc/adapters.h) and the kernel of the product: what test_adapters_ways_cpu.py looks up and
test_gpu_adapters_ways.py runs."""
import paper_2210_12415_amd as alt

BF16, F32 = alt.BF16, alt.F32
# way, the product's kernel ("any": operands at any alignment, by the tiles; "packed": they are laid out anew first; "few": its column tiles, parts of its reduction and
# of the inner sums'), type, M, N, K, adapters, rank
WAYS = [
    ("few", "1 1 1", BF16, 17, 64, 64, 3, 200), ("few", "1 1 2", BF16, 22, 64, 320, 8, 4), ("few", "1 1 8", BF16, 32, 4096, 4096, 24, 16), ("few", "1 4 8", BF16, 32, 512, 8192, 24, 16), ("few", "2 1 1", BF16, 65, 3520, 64, 40, 64),
    ("few", "1 1 1", BF16, 5, 1031, 130, 4, 16), ("few", "1 2 1", F32, 37, 128, 1984, 8, 200), ("few", "2 1 2", F32, 70, 3966, 145, 64, 4), ("few", "1 1 2", F32, 333, 515, 1030, 5, 7),
    ("beside", "deep", BF16, 309, 2560, 1856, 40, 4), ("beside", "half", BF16, 2328, 640, 896, 40, 16), ("beside", "middle", BF16, 800, 4096, 512, 64, 4),
    ("beside", "large", BF16, 3561, 2624, 640, 64, 4), ("beside", "any 128", BF16, 5698, 270, 2174, 40, 16), ("beside", "any 64", BF16, 162, 3790, 2550, 40, 16),
    ("beside", "packed", BF16, 1100, 4090, 4095, 64, 4), ("beside", "ring", F32, 100, 1000, 16384, 40, 16),
    ("fused", "deep", BF16, 1350, 64, 64, 1, 200), ("fused", "shallow", BF16, 1298, 1536, 128, 3, 64), ("fused", "half", BF16, 1219, 832, 64, 8, 33), ("fused", "middle", BF16, 663, 3136, 72, 3, 33),
    ("fused", "large", BF16, 2477, 3264, 64, 1, 4), ("fused", "any 128", BF16, 2100, 1030, 1031, 6, 16), ("fused", "any 128", BF16, 838, 2430, 69, 3, 7),
    ("fused", "any 64", BF16, 1500, 700, 129, 3, 16), ("fused", "any 64", BF16, 41, 2615, 65, 3, 200), ("fused", "packed", BF16, 2100, 2050, 2047, 6, 16),
    ("fused", "ring", F32, 235, 384, 64, 1, 200), ("fused", "any 64", F32, 34, 2597, 91, 3, 200), ("fused", "any 64 many", F32, 2507, 794, 106, 40, 16),
]
