"""4-bit weights on the host: the layout of the paged tensor, byte by byte, and
the product in 64 bits with the bound of its rounding errors."""
import numpy as np
import torch


def sizes(rows, cols, group):
    """Row tiles, column segments, groups of a segment."""
    return -(-rows // 16), -(-cols // 128), 128 // group


def packed(codes, scales, zeros, group):
    """The tensor's bytes from codes [rows, cols] (uint8) and 16-bit patterns of
    scales and zeros [rows, cols / group] (uint16; zeros may be None)."""
    rows, cols = codes.shape
    tiles, segs, per = sizes(rows, cols, group)
    out = np.zeros(tiles * segs * 1024, dtype=np.uint8)
    for m in range(rows):
        for k in range(cols):
            block, r, c = m // 16 * segs + k // 128, m % 16, k % 128
            word, g, e = c // 32, c % 32 // 8, c % 8
            bit = 4 * (e // 2 + 4 * (e % 2))
            out[block * 1024 + (g * 16 + r) * 16 + word * 4 + bit // 8] |= (codes[m, k] & 15) << (bit % 8)
    planes = [out]
    for t in (scales, zeros):
        if t is None:
            continue
        p = np.zeros(tiles * segs * per * 16, dtype=np.uint16)
        for m in range(rows):
            for j in range(cols // group):
                block, r = m // 16 * segs + j // per, m % 16
                p[block * per * 16 + (r // 4 * per + j % per) * 4 + r % 4] = t[m, j]
        planes.append(p.view(np.uint8))
    return np.concatenate(planes)


def product(codes, scales, zeros, group, x):
    """y [batch, rows] in 64 bits, and the bound of the kernel's error.

    All products are exact in fp32.  A group's sum begins with at most 128
    additions of (8 + 16) x (or x, times a rounded 16 + z, with zero points) and goes on
    with 128 of (n + 16) x; each is one rounding of at most the magnitudes'
    sum, 2^-24 of it.  Scaling and adding up: two roundings a group and the sum
    over the groups and wavefronts, of the partial sums so far."""
    n = torch.from_numpy(codes.astype(np.float64))
    s, z = scales.double(), torch.full(scales.shape, 8.0, dtype=torch.float64) if zeros is None else zeros.double()
    wide = lambda t: t.repeat_interleave(group, 1)  # noqa: E731
    xs = x.double()
    y = xs @ (wide(s) * (n - wide(z))).T
    # (-0 in the sums, sign of s: magnitudes only)
    mass = xs.abs() @ (wide(s.abs()) * (n + 16 + wide(z.abs()) + 16)).T
    groups = scales.shape[1]
    depth = 2 * 128 + 4 + groups + 8
    return y, depth * 2.0 ** -24 * mass
