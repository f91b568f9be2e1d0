"""Layers with weights by group whose last tiles come in parts, or whose weight gradients do: rows of every group, widths."""

TAILS = [([2600, 0, 1100, 700, 1], 4096, 4104),        # 340 tiles of Z, 84 of them in three parts; 320 of dX
         ([6000, 5000, 0, 4000, 300], 2056, 4104),     # 1054 of Z, 30 in eight parts of 320 indices, the last one of none
         ([6000, 5000, 0, 4000, 300], 4104, 2056),     # the same of dX
         ([8003, 3], 4096, 4104),                      # 561: 49 in five parts
         ([700] * 8 + [1], 8200, 3080)]                # 325 of Z; 825 of dX, 57 in four parts


def many_lengths(n, groups):
    """Of no row, of a few, of several tiles; n in all."""
    lens = [(0, 1, 256, 700, 0, 300, 257, 2000, 513, 900)[(i * i + i // 7) % 10] for i in range(groups)]
    lens[-1] += n - sum(lens)
    assert lens[-1] >= 0
    return lens


MANY = [(300_000, 520, 1024, 512)]

JOINED = [([700, 0, 701, 99, 1500], 33, 65), ([3000, 1, 2999], 7, 9), ([900, 1100, 800], 26, 33), ([2000, 2000], 5, 15)]
