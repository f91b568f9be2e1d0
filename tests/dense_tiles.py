"""Layers whose products run in the dense kernel's larger tiles: sizes, and the tile and parts of the contraction that Z, dX and dW take
(csrc/dense_plan.hpp; the host test compares them with it, so that a change of its costs does not leave a tile without a test).

`whole`: rows of X, W and the gradient are whole 16-byte pieces.  Every case has a remainder in each side of the tiles it is there for, and
an end of the contraction inside a step."""

#       n      d_in  d_out fp32   whole  tile and parts of Z, dX, dW
CASES = [
    (3333, 136, 2312, False, True, (256, 1), (64, 3), (64, 4)),
    (3333, 2312, 136, False, True, (64, 3), (256, 1), (64, 4)),
    (137, 3336, 2312, False, True, (64, 4), (64, 3), (256, 1)),
    (2056, 4104, 2056, False, True, (256, 3), (256, 1), (256, 1)),
    (2900, 72, 1032, False, True, (128, 1), (64, 1), (64, 12)),
    (2900, 1032, 72, False, True, (64, 1), (128, 1), (64, 12)),
    (19997, 776, 776, False, True, (128, 1), (128, 1), (128, 10)),
    (3333, 333, 1537, False, False, (128, 1), (64, 1), (64, 5)),
    (3333, 1537, 333, False, False, (64, 1), (128, 1), (64, 5)),
    (333, 3333, 1537, False, False, (64, 5), (64, 1), (128, 1)),
    (2900, 72, 1028, True, True, (128, 1), (64, 5), (64, 12)),
    (2900, 1028, 72, True, True, (64, 5), (128, 1), (64, 12)),
    (75, 2900, 1028, True, True, (64, 12), (64, 5), (128, 1)),
    (1793, 1032, 324, True, True, (128, 5), (64, 1), (64, 5)),
    (2561, 35, 1537, True, False, (128, 1), (64, 7), (64, 41)),
    (2561, 1537, 35, True, False, (64, 7), (128, 1), (64, 41)),
    (37, 2561, 1537, True, False, (64, 41), (64, 7), (128, 1)),
]
