"""The products with 4-bit weights in 64 bits and the bound that follows from the order
in which the kernel adds.

A group's columns are added in the matrix cores' fp32 accumulator, one rounding a
column and part at most, of partial sums that are at most the sum of all terms'
sizes.  With codes that carry an offset, taken out by a product of its own, a term would be
|x| times up to 2 offset + 15.  The group's sum times its scale is added to a
wave's sum (two roundings a group of its tiles, with the row scale of 8 bits a third), and
up to 16 waves' sums to the output's.  Products of two 16-bit numbers are exact in fp32.
"""
import numpy as np

U = 2.0 ** -24


def split_sums(x, weights, scales, group):
    """Of each output and group: the sum of x (code - 8) and of |x|, times |scale|,
    and |scale| |sum|: arrays [M][rows] summed over the groups."""
    M, K = x.shape
    y = np.zeros((M, weights.shape[0]))
    size, sums = np.zeros_like(y), np.zeros_like(y)
    for g in range(scales.shape[1]):
        a, e = g * group, min((g + 1) * group, K)
        s = x[:, a:e] @ weights[:, a:e].T
        y += s * scales[:, g]
        size += np.abs(x[:, a:e]).sum(1, keepdims=True) * np.abs(scales[:, g])
        sums += np.abs(s * scales[:, g])
    return y, size, sums


def product(x, weights, scales, group, parts, offset):
    """(y, bound): weights codes less 8, [rows][K]; scales [rows][groups]; parts: 16-bit
    numbers that a value of x is cut into; offset: what is added to a code."""
    y, size, sums = split_sums(x, weights, scales, group)
    K = x.shape[1]
    tiles = -(-K // 128)
    waves = min(tiles, 16)
    groups = -(-tiles // waves) * (128 // group)      # of a wave
    largest = 8 if offset == 0 else (offset + 7) + (offset + 8)
    per_group = group * (parts + (1 if offset else 0))
    return y, U * (per_group * largest * size + (2 * groups + waves + 3) * sums)
