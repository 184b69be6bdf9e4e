"""Philox4x32-10 by the paper's definition, and its published test vectors."""

# (counter words, key words, result words)
VECTORS = [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
]


def words(counter, key):
    """Four words of a counter: a round multiplies words 0 and 2 and exchanges the halves of the products."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [p1 >> 32 ^ c[1] ^ k[0], p1 % 2 ** 32, p0 >> 32 ^ c[3] ^ k[1], p0 % 2 ** 32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return tuple(c)


def halves(chunk, seed, offset, site):
    """The 16 random bits of the eight elements of a dropout's chunk."""
    w = words((chunk, site, offset % 2 ** 32, offset >> 32), (seed % 2 ** 32, seed >> 32))
    return [h for x in w for h in (x & 0xFFFF, x >> 16)]
