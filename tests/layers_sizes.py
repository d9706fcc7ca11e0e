"""Sizes of the layers before the head that take each of their kernels: what tests/test_gpu_linear_kernels.py and tests/test_gpu_rms_kernels.py run, and what
tests/test_layer_launches.py sees launched.  A product's: rows, width, outs, options of test_gpu_linear.case; what is launched, "join" among it or not."""

BIG, MID, FEW = "Cfg<256, 256,", "Cfg<128, 128,", "Cfg<128, 64,"
JOIN = "k_linear_join"

# 256 x 256 tiles: whole ones and, at the end of the outs, some of 64 or 128 x 256; all whole; shared by several workgroups at the end
LARGEST = {
    "64 at the end": (2048, 1024, 4100, dict(pad=4)),
    "128 at the end": (2040, 520, 4456, dict()),
    "whole": (4096, 1024, 4096, dict()),
    "shared": (4096, 4096, 4100, dict(pad=4)),
}
LARGEST_8 = {
    "64 at the end": (2048, 2048, 4100, dict(pad=4, bits=8)),
    "128 at the end": (2040, 1000, 4456, dict(bits=8)),
}

# up to 32 rows, the weight straight into registers: fragments of outs, of rows, steps at a time, waves
THIN = {
    "1, 1, 2, 16": [(1, 512, 4000), (16, 77, 300)],
    "1, 1, 2, 8": [(1, 200, 4100), (16, 1000, 8100)],
    "1, 1, 2, 4": [(1, 1000, 8200), (13, 77, 8195), (16, 4096, 11000)],
    "1, 2, 2, 8": [(17, 200, 1000), (32, 1030, 6128)],
    "2, 2, 2, 8": [(17, 1000, 6150), (32, 77, 10000)],
    "4, 2, 2, 8": [(32, 200, 10240), (19, 4096, 11001), (17, 77, 10250)],
}

# 33 to 64 rows, tiles whose k several workgroups share: (6 a tile, 16, 8)
FEW_SHARED = [(64, 4096, 5000), (48, 4096, 1100), (33, 2048, 2500)]

# gradients in unshared whole 256 x 256 tiles: of x, of the weight, of both
GRADS = {"d_x": (4096, 4096, 1024), "d_weight": (1024, 4096, 4096), "both": (4096, 4096, 4096)}

# rows in 8 bits that a workgroup takes one after the other, of two, three and four pieces a lane: the last of them of eight elements, of one, a full one
RMS_AHEAD = [(4609, 2056), (4609, 5121), (4096, 8192)]
# gradients of rows that are loaded when the one before is done
RMS_GRADS_RELOAD = [(600, 8200), (513, 16390), (600, 32768)]
