"""Sizes that take the layers' matrix-core products through every tile shape and every way of cutting them, and a look at the choice."""
import ctypes as C

from paper_2010_01546_amd import binding as b


class TileChoice(C.Structure):
    """struct TileChoice of the sources"""
    _fields_ = [(n, C.c_int) for n in ("few", "rows", "columns", "whole", "cut", "runs", "stages")]


def choice(product, dt, N, M, S):
    """product: "forward", "dX", "dW" or "int8" """
    c = TileChoice()
    if product == "int8":
        b.lib._ZN2fw10int8_tilesEiiiPNS_10TileChoiceE(N, M, S, C.byref(c))
    else:
        b.lib._ZN2fw11gated_tilesEi8fw_dtypeiiiPNS_10TileChoiceE(("forward", "dX", "dW").index(product), dt, N, M, S, C.byref(c))
    return c


def way(c):
    """("rows x columns", how cut), or None for few rows and for contractions of one or two stages."""
    if c.few or c.stages < 3:
        return None
    return f"{c.rows}x{c.columns}", "both" if c.whole and c.cut else "runs" if c.cut else "whole"


BF16_SIZES = [(129, 575, 65), (8545, 513, 129), (2899, 3053, 65), (129, 266, 2923), (517, 545, 6559), (139, 4159, 1865), (5575, 5939, 65), (195, 8603, 207),
              (1417, 8319, 67), (6529, 591, 603), (335, 5497, 709), (5422, 650, 418), (196, 8720, 979), (8299, 741, 69), (129, 465, 11039), (259, 267, 10131),
              (137, 8298, 3606), (7947, 572, 1798), (555, 7387, 591), (5035, 909, 1573), (8491, 7071, 195), (2504, 900, 3209), (385, 4997, 9359)]
F32_SIZES = [(139, 131, 69), (1107, 261, 65), (2119, 1549, 65), (193, 387, 4701), (131, 2883, 1520), (8412, 407, 71), (8431, 137, 339), (707, 8341, 73),
             (1903, 655, 1557), (267, 387, 6457), (6061, 4237, 65), (391, 8275, 67), (518, 7857, 66), (135, 195, 10943), (485, 989, 8311)]
INT8_SIZES = [(129, 575, 65), (2899, 3053, 65), (517, 545, 6559), (139, 4159, 1865), (6529, 591, 603), (8299, 741, 69), (137, 8298, 3606), (7947, 572, 1798),
              (5035, 909, 1573), (2504, 900, 3209), (8257, 8931, 131), (1413, 947, 10977), (385, 4997, 9359), (134, 22007, 8405), (8545, 513, 129), (5575, 5939, 65),
              (5422, 650, 418), (8491, 7071, 195)]
