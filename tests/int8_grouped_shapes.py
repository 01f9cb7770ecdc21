"""Sizes at which products of 8-bit integers and of grouped rows run in every form that they have."""

# (m, n, k): each tile, whole and with its contraction split, with outputs that leave as whole lines and ones that do not, up to
# 1024 outputs a row (which one workgroup joins from the parts) and more, over several rounds of the pipeline.
INT8 = [(2883, 130, 19824), (147, 5546, 13856), (5567, 152, 14080), (129, 6136, 13888), (8357, 905, 688), (422, 17428, 528),
        (8366, 936, 640), (259, 22048, 544), (2161, 66, 15296), (68, 2332, 16928), (4212, 72, 9824), (69, 2072, 16384),
        (6779, 270, 560), (69, 17191, 592), (8222, 208, 544), (65, 17136, 512), (65, 527, 18448), (5, 4477, 3984),
        (65, 584, 16992), (5, 1032, 16368), (8687, 67, 544), (5, 16554, 528), (8395, 72, 512), (5, 19248, 528), (5, 19, 4272),
        (5, 1094, 4224), (5, 16, 4000), (5, 1072, 4048), (5, 17, 592), (6, 1044, 512), (6, 16, 512), (5, 1136, 528)]

# (rows of each group, n, k, block), forward.  The kernels for few rows: 16 and 32 rows, 64 and 128 weight rows.
FEW = [([9, 12] * 16, 2056), ([3, 0, 16], 48), ([24, 27, 30, 17] * 8, 2056), ([32, 1, 0, 33] * 8 + [32] * 12, 2051), ([30, 25], 40),
       ([60, 40, 0], 130)]
FEW_INNER = [(16, 16), (256, 16), (272, 16), (512, 16), (528, 16), (768, 16), (1024, 16), (1040, 16), (1280, 16), (96, 32), (288, 32),
             (1152, 32), (64, 64), (832, 64), (1280, 64), (128, 128), (640, 128), (1024, 128)]
GROUPED = [(sizes, n, k, block) for sizes, n in FEW for k, block in FEW_INNER]

# The largest tile: (inner, blocks), 64, 128 and 256 rows of it, by their first and last columns.
TALL, TALL_OUTER = [300, 600, 513, 130, 380, 256], 8192
TALL_INNER = [(block * count, block) for block in (32, 64, 128) for count in (1, 3, 4, 5, 8)]
