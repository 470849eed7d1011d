"""Lists of matrices that take each of the products' kernels, ragged and both
tall and wide: {name: (shapes, kernels with PRODUCTS_F32, with PRODUCTS_F16)}, the
kernels as (side, groups of waves) of the three products and the parts of a Gram
tile's sum.  A change of what the sizes lead to shows here, and these lists
have to follow it so that every kernel stays covered."""


def _all(side, groups):
    return dict(gram=(side, groups), poly=(side, groups), next=(side, groups), parts=1)


KERNEL_LISTS = {
    "64 by two groups": ([(300, 200), (130, 500)], _all(64, 2), _all(64, 2)),
    "64 by four groups": ([(950, 1020)], _all(64, 4), _all(64, 4)),
    "64 by four groups, tall": ([(1020, 950)], _all(64, 4), _all(64, 4)),
    "128": ([(700, 900), (900, 650)] * 8, _all(128, 1), _all(128, 1)),
    "256": ([(464, 517), (517, 464)] * 39, _all(256, 1), _all(256, 1)),
    "256, halves": ([(1000, 1100), (1100, 1000)] * 24, _all(128, 1), _all(256, 1)),
    "128 padded to 256": (
        [(2000, 2040), (2040, 1999)] * 8,
        dict(gram=(128, 1), poly=(128, 1), next=(256, 1), parts=1),
        dict(gram=(128, 1), poly=(128, 1), next=(256, 1), parts=1)),
    "long sums in parts": (
        [(17, 9000), (9000, 30)],
        dict(gram=(64, 4), poly=(64, 2), next=(64, 2), parts=18),
        dict(gram=(64, 4), poly=(64, 2), next=(64, 2), parts=9)),
    "parts, padded to 128": (
        [(72, 1256), (1256, 70)] * 8,
        dict(gram=(64, 4), poly=(64, 2), next=(128, 1), parts=3),
        dict(gram=(64, 2), poly=(64, 2), next=(128, 1), parts=1)),
}
