"""Sizes (M, K, N) whose weight's gradient from 8 bits goes through the steady loop of its
kernel on 256 compute units, and what the call launches: parts of five whole stages of 32
rows and more, in whole tiles.  The GPU tests run them, and a CPU test asserts that the
calls are cut so."""
STEADY = [
    ((1250, 768, 1280), "8-bit tiles of 128, 240 workgroups, 4 splits"),
    ((2600, 512, 640), "8-bit tiles of 128, 240 workgroups, 12 splits"),
    ((3000, 384, 512), "8-bit tiles of 128, 192 workgroups, 16 splits"),
    ((1500, 1300, 1100), "8-bit tiles of 128, 396 workgroups, 4 splits"),
]


def stages(M, line):
    """Stages of 32 rows in a part, of a launch's line."""
    return -(-(-(-M // 32)) // int(line.split()[-2]))
