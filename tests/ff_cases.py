"""Sizes that take the 256 x 256 tiles on 256 compute units: the GPU tests run
them, and a CPU test asserts which kernels their calls launch."""
# (M, K, N), what the forward call launches, what the gradient's dx and dw launch
LARGE_TILES = [
    ((4000, 520, 4008), ["direct tiles of 256, 256 workgroups, 1 splits"], None),
    ((4000, 72, 4008), ["direct tiles of 256, 256 workgroups, 1 splits"], None),
    ((3000, 2000, 3008), ["direct tiles of 256, 144 workgroups, 1 splits"],
     ["direct tiles of 256, 192 workgroups, 2 splits"] * 2),
    ((2056, 4008, 4104), ["direct tiles of 256, 153 workgroups, 1 splits"],
     ["direct tiles of 256, 144 workgroups, 1 splits", "direct tiles of 256, 272 workgroups, 1 splits"]),
]
