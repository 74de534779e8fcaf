"""Batches that keep the rings in LDS turning: one for every kernel that a product of codes or a gradient may take, with random codes and so
many steps that places are loaded again at least twice, tiles with an even and with an odd number of stages.  The library's own rules,
compiled for the host, say which kernel a batch takes (tests/test_linear_choice.py holds them to it)."""
import ctypes
import functools
import os
import subprocess
import tempfile
from typing import NamedTuple

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2509_09679_amd", "csrc")


class Kernel(NamedTuple):
    few: int     # rows: blocks x cols pieces of 16 x 16, alone on a compute unit or not; else a tile
    blocks: int
    cols: int
    alone: int
    tile: int
    across: int  # weights of a gradient as they lie


class Choice(NamedTuple):
    kernel: Kernel
    waves: int   # that share the sum
    depth: int   # places of a ring
    codes: int   # of a stage or step


@functools.lru_cache(None)
def _rules():
    with tempfile.TemporaryDirectory() as d:
        so = os.path.join(d, "linear_choice.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, os.path.join(HERE, "linear_choice.cpp"), "-o", so], check=True)
        return ctypes.CDLL(so)


def _choice(name, rows, *args):
    out = (ctypes.c_int * 9)()
    getattr(_rules(), name)(ctypes.c_int64(rows), *args, out)
    return Choice(Kernel(*out[:6]), *out[6:])


def forward_choice(T, N, K, experts, xbits, wbits):
    """Of rows that are whole 16-byte pieces; experts: 0 for a call that is not grouped."""
    return _choice("linear_forward_choice", T, K, N, experts, xbits, wbits)


def gradient_choice(T, N, K, experts, wbits, terms, aligned=True):
    return _choice("linear_gradient_choice", T, N, K, experts, wbits, terms, int(aligned))


def steps(choice, summed):
    """(stages of a tile or steps of all waves, steps of the wave that has the fewest)"""
    n = -(-summed // choice.codes)
    return n, n // choice.waves


# (xbits, wbits): tokens, outputs, inputs, experts
FORWARD = {
    (8, 8): [(1, 1, 6144, 0), (37, 4947, 4416, 0), (61, 11661, 672, 3), (75, 3283, 2112, 0), (109, 7435, 576, 5), (468, 9337, 576, 5),
             (772, 9983, 448, 5), (868, 8327, 576, 5), (1410, 707, 832, 0), (1427, 5512, 416, 0), (2059, 1, 4352, 5),
             (2258, 2318, 480, 16), (2831, 20, 5120, 0), (3393, 20, 2496, 3), (4724, 65, 2496, 0), (5155, 167, 672, 16),
             (5220, 18, 4320, 0), (5261, 18, 1984, 5), (5474, 1, 2560, 3), (5816, 1, 6080, 0), (5819, 1184, 576, 16)],
    (8, 4): [(1, 1, 5056, 0), (151, 7439, 800, 5), (172, 11597, 704, 2), (1166, 6300, 800, 2), (1774, 3697, 672, 16),
             (1868, 3632, 576, 16), (1917, 103, 2592, 16), (2614, 17, 4192, 3), (4118, 332, 640, 0), (4723, 70, 2080, 0),
             (5370, 233, 672, 2), (5538, 1172, 672, 16), (5621, 17, 2592, 2), (5771, 1, 4032, 3)],
    (8, 2): [(1, 1, 8128, 0), (180, 6647, 704, 5), (203, 8997, 832, 3), (333, 11867, 704, 5), (547, 11816, 832, 5), (721, 9905, 704, 5),
             (968, 6305, 832, 5), (1178, 1128, 704, 0), (2553, 20, 4992, 0), (4807, 33, 4160, 16), (5049, 268, 832, 0),
             (5279, 66, 4224, 0), (5614, 22, 3968, 5), (5842, 1, 4032, 5)],
    (4, 8): [(2, 1, 6048, 0), (34, 5202, 960, 0), (35, 6127, 2016, 0), (45, 2565, 6720, 0), (75, 1779, 4128, 0), (117, 7421, 672, 5),
             (458, 11386, 576, 3), (535, 2094, 800, 16), (2242, 1, 5184, 3), (2897, 2411, 672, 5), (3045, 356, 800, 5),
             (4259, 66, 2144, 3), (4263, 65, 4096, 0), (4787, 237, 672, 0), (5215, 1, 6176, 0), (5384, 17, 2496, 5), (5499, 1302, 576, 2),
             (5716, 1300, 672, 3), (5873, 19, 5184, 0), (5895, 1, 4128, 2)],
    (4, 4): [(1, 1, 6048, 0), (89, 11628, 832, 3), (102, 2086, 4096, 2), (174, 6773, 672, 5), (598, 8788, 672, 5), (1984, 51, 5600, 16),
             (2122, 737, 672, 0), (3799, 385, 800, 5), (4407, 67, 2496, 5), (5283, 17, 4224, 0), (5590, 1, 5088, 0), (5946, 1291, 832, 0)],
    (4, 2): [(1, 1, 10176, 0), (78, 2491, 4928, 2), (166, 6936, 896, 5), (294, 433, 8448, 0), (503, 2113, 704, 16), (1195, 5928, 832, 2),
             (1556, 3139, 704, 16), (4458, 68, 4224, 5), (5358, 17, 5120, 0), (5578, 1, 9216, 0), (5620, 279, 704, 0), (5794, 259, 832, 5)],
}

# (terms, wbits): tokens, outputs, inputs, experts
GRADIENT = {
    (2, 2): [(48, 419, 3584, 16), (55, 383, 3584, 16), (83, 393, 7744, 2), (168, 364, 4608, 3), (407, 327, 8256, 3), (496, 398, 9408, 2),
             (899, 411, 4544, 3), (3332, 322, 1728, 16), (3689, 2428, 36, 0), (5684, 274, 784, 16), (5751, 396, 656, 3)],
    (2, 4): [(33, 389, 3808, 16), (69, 323, 7808, 2), (92, 387, 6944, 2), (482, 404, 8512, 0), (673, 321, 4352, 3), (683, 406, 7232, 2),
             (2307, 2114, 38, 0), (2899, 1490, 18, 3), (3102, 2861, 18, 0), (4207, 137, 208, 0), (4992, 340, 176, 0), (5243, 329, 704, 16),
             (5558, 328, 672, 2), (5681, 340, 928, 16)],
    (2, 8): [(1, 3021, 8, 0), (4, 260, 8384, 3), (18, 411, 3488, 16), (23, 334, 1568, 16), (72, 333, 3472, 16), (102, 336, 7680, 0),
             (246, 401, 2784, 3), (851, 417, 4384, 2), (1044, 2181, 17, 3), (1367, 194, 675, 0), (2432, 972, 45, 2), (2437, 323, 2432, 0),
             (3899, 265, 229, 3), (4995, 344, 688, 16), (5076, 396, 720, 2), (5147, 332, 720, 0), (5385, 270, 784, 16),
             (5859, 332, 800, 16), (5891, 962, 17, 3)],
    (3, 2): [(2, 1990, 8, 0), (110, 321, 6336, 0), (422, 418, 1536, 5), (2225, 268, 704, 16), (2358, 1119, 8, 2), (5330, 322, 112, 0),
             (5781, 331, 320, 16), (5968, 194, 272, 0)],
    (3, 4): [(142, 403, 4864, 0), (1875, 270, 1056, 5), (4099, 322, 448, 16), (4919, 325, 160, 16), (5230, 387, 106, 16),
             (5462, 258, 272, 0)],
    (3, 8): [(161, 392, 4032, 0), (324, 199, 4992, 2), (509, 258, 3248, 3), (2607, 1224, 18, 2), (2879, 2047, 18, 0), (3026, 471, 42, 0),
             (4463, 359, 144, 16)],
}

FORWARD_CASES = [(*c, *bits) for bits, cases in FORWARD.items() for c in cases]
GRADIENT_CASES = [(*c, wbits, terms) for (terms, wbits), cases in GRADIENT.items() for c in cases]
