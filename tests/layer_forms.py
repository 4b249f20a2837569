"""Sizes that reach every kernel of the layers by role, in 8-bit integers and from kept bytes, next to those of their own tests."""


def spread(n, groups, most):
    """`groups` sizes that add up to n: one of `most`, some of none, one or a few rows, the rest alike."""
    few = [0, 1, 5][:max(groups - 2, 0)]
    rest, left = groups - 1 - len(few), n - most - sum(few)
    return [*few, *([left // rest] * (rest - 1) + [left - left // rest * (rest - 1)] if rest else []), most]


# sizes of the groups, d_in, d_out
GROUPED = [
    ([60_000, 3, 71_098], 256, 256),                          # 256 x 256 tiles of the weights' gradient, shares across groups
    (spread(131_101, 12, 40_000), 400, 496),                  # and where they end inside a tile
    (spread(140_003, 64, 9_000), 528, 512),                   # many groups end inside the large tiles
    ([131_099, 1], 2064, 2064),                               # more tiles than workgroups
    ([131_100], 4368, 4112),                                  # one share, no second launch
    (spread(20_000, 40, 3_000), 256, 256),                    # 128 x 128 tiles by group, several units a group
    ([200] * 40, 272, 256), ([5] * 60, 272, 256),             # and one unit a group
    (spread(30_000, 80, 5_000), 512, 64), ([100] * 80, 512, 64), ([3] * 140, 512, 64),      # 256 x 64 tiles by group
    (spread(70_001, 4, 30_000), 1024, 64),                    # and shares
    ([300, 0, 401], 4096, 4112),                              # 128 x 128 tiles, one share
    (spread(33_717, 46, 2_000), 80, 80),                      # large float32 tiles by group
    (spread(72_830, 83, 9_000), 208, 80), (spread(40_000, 3, 39_000), 1024, 1040),
    (spread(530_001, 5, 100_000), 32, 64),                    # many shares of few values
    # many groups beside what the units' rows go into all of them: only groups of two units or more have places in the workspace
    (spread(10_007, 100, 4_000), 160, 1040), (spread(2_400, 60, 1_500), 16, 32), (spread(9_300, 78, 7_000), 32, 16),
    (spread(131_100, 16, 90_000), 2064, 2064), (spread(10_110, 203, 4_000), 352, 48), (spread(17_000, 100, 9_000), 4096, 48),
    ([1_000, 1_500, 7] * 60, 1024, 1024), ([0, 3, 600, 1] * 64, 512, 512), ([1] * 200 + [2_600] * 2 + [0] * 54, 64, 256),
    ([2_000, 2_608], 16, 16), (spread(140_000, 30, 60_000), 16, 16),
]
# n, d_in, d_out
PACKED = [(301, 4096, 4112), (131_075, 2832, 2816), (131_093, 256, 256), (131_101, 400, 496), (140_003, 528, 512), (131_089, 2064, 2064), (40_003, 48, 1024),
          (1_001, 112, 4112), (70_001, 1024, 64), (20_011, 160, 16), (140_001, 80, 272), (35_656, 80, 80), (66_001, 400, 80)]
INT8 = [(66_001, 272, 400), (131_073, 528, 160), (262_139, 272, 1040), (33_003, 80, 144)]
