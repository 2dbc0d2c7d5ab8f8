"""Test infrastructure: sizes of linear layers that together reach every kernel on the matrix cores, with ragged ends in every direction.  test_layers_dispatch_of_linear.py holds that they do, test_layers_values_gpu.py
compares their results."""

# tokens, outs, cols, values between rows
LINEAR = [
    (13, 141, 78, 0),       # tiles of 64 x 64, or 128 x 64 in fp32
    (14, 156, 219, 0),      # two teams of wavefronts
    (12, 159, 1470, 3),     # and several parts
    (76, 8614, 65, 1),      # 128 x 64
    (74, 8431, 196, 0),
    (70, 3000, 4100, 0),
    (4690, 428, 78, 0),     # 128 x 128
    (840, 2317, 2441, 0),
    (2709, 262, 867, 1),
    (6922, 1675, 1310, 0),  # 256 x 256, rows that begin anywhere
    (5778, 4984, 1344, 1),
    (3900, 4090, 1600, 0),  # the same straight to LDS, where outs allow it
    (4000, 4088, 1472, 0),
    (5778, 4984, 1344, 0),  # more tiles than there are workgroups
]
