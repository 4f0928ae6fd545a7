"""Calls that reach every kernel of the 4-bit linears; the host tests check that they do."""

# (rows of A, tiles of 16 columns a wave, waves along K, along the columns, stages): rows and columns that take it
VARIANTS = {
    (8, 1, 8, 1, 3): (3, 70), (16, 1, 8, 1, 3): (11, 2500), (8, 2, 8, 1, 2): (3, 5000), (16, 2, 8, 1, 2): (11, 5000),
    (8, 1, 4, 1, 3): (3, 9000), (8, 2, 4, 1, 3): (3, 14000), (8, 2, 4, 1, 2): (3, 17000), (16, 2, 4, 1, 2): (11, 9000),
    (16, 4, 4, 1, 2): (11, 17000), (16, 4, 2, 2, 3): (11, 33011), (32, 1, 4, 2, 3): (27, 4500), (32, 2, 4, 2, 3): (50, 4500),
    (32, 1, 2, 4, 3): (27, 17000), (32, 4, 2, 2, 2): (27, 33011), (64, 1, 2, 4, 3): (50, 14000), (64, 1, 1, 4, 3): (50, 17000),
    (64, 1, 1, 8, 3): (50, 33011)}


def panel(v):
    """Steps of 128 k whose scales a workgroup of the variant holds at a time."""
    return 256 // {1: 1, 2: 2, 4: 4, 8: 8}[v[1] * v[3]]


def beyond_panels():
    """(variant, M, N, K): a second panel of scales of three steps and a piece (waves without a step where more share K), and a
    third one behind a whole second of more columns than rows of the ring (where the weights stay below 200 MB)."""
    out = []
    for v, (M, N) in VARIANTS.items():
        out.append((v, M, N, (panel(v) + 3) * 128 + 32))
        K = (2 * panel(v) + v[2] * v[4] + 1) * 128 + 96
        if N * K < 400_000_000:
            out.append((v, M, N, K))
    return out


# N, K and numbers of rows of A that one variant serves
ROWS = [
    (300, 4128, (8, 1, 8, 1, 3), (1, 7, 8)), (2500, 1056, (16, 1, 8, 1, 3), (9, 12, 16)), (6144, 4128, (8, 2, 8, 1, 2), (1, 5, 8)),
    (6144, 4128, (16, 2, 8, 1, 2), (9, 10, 16)), (6144, 4128, (32, 1, 4, 2, 3), (17, 25, 32)), (6144, 4128, (32, 2, 4, 2, 3), (33, 50, 64)),
    (6144, 4128, (64, 1, 2, 4, 3), (65, 80, 128)), (9000, 1056, (8, 1, 4, 1, 3), (1, 8)), (9000, 1056, (16, 2, 4, 1, 2), (9, 16)),
    (14000, 1056, (8, 2, 4, 1, 3), (1, 3, 8)), (17000, 1056, (8, 2, 4, 1, 2), (1, 8)), (17000, 1056, (16, 4, 4, 1, 2), (9, 16)),
    (17000, 1056, (32, 1, 2, 4, 3), (17, 32)), (17000, 1056, (64, 1, 1, 4, 3), (33, 64)), (17000, 1056, (64, 1, 1, 8, 3), (65, 100, 128)),
    (33011, 1056, (16, 4, 2, 2, 3), (9, 16)), (33011, 1056, (32, 4, 2, 2, 2), (17, 32)),
]
