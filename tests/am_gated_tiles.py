"""Sizes (rows, inner, results) of gated layers whose dense operands each kernel of the tiled forward takes, with the kernel
for 16-bit operands and for 8-bit ones.  test_am_gated_tiles.py holds them to the plan, test_gpu_am_gated_tiles.py runs them."""

SIZES = {
    (2904, 144, 1500): ("256", "256"),
    (2500, 64, 1540): ("256", "256"),
    (1470, 336, 2040): ("128 x 256", "128 x 256"),
    (1921, 80, 1913): ("128 x 256", "128 x 256"),
    (2040, 464, 980): ("128, one a CU", "128, one a CU"),
    (900, 336, 1100): ("128, one a CU", "128, one a CU"),
    (66000, 64, 33): ("128", "128"),         # few results for very many rows
    (700, 16, 1000): ("64", "64"),
    (700, 48, 1000): ("64", "64"),
    (700, 144, 1000): ("64", "64"),
    (1470, 328, 2040): ("128 x 256", "128, staged"),
    (1500, 333, 1200): ("128, staged", "128, staged"),
    (1501, 77, 1203): ("128, staged", "128, staged"),
}
# shorter than a fetch, at its ends and at a stage's ends
SIZES.update({(700, k, 1000): ("64, staged", "64, staged") for k in (1, 7, 9, 15, 17, 63, 65, 127, 129, 145)})
SIZES.update({(700, k, 1000): ("64", "64, staged") for k in (8, 24, 72)})
