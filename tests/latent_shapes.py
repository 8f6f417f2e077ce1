"""Batches that take each way through the absorbed latent attention on a device of 256 compute units, and what the plan
has to say of them: the host's test holds the plans to it, the device's tests run the batches.

name: (heads, cached, new, row tile, dealt by tile, least units of the longest share)
"""


def _spread(least, step, count):
    return [least + step * r for r in range(count)]


ROUTES = {
    # few rows: the waves of a workgroup divide the key tiles
    "rows16": (8, [700, 40], [1, 2], 16, 1, 4),
    "rows16_long": (16, _spread(15000, 37, 40), [1] * 40, 16, 0, 65),      # more than 16 tiles to each of four waves
    "rows32": (16, [600, 33], [2, 1], 32, 1, 4),
    "rows32_two_waves": (28, _spread(1000, 97, 32), [1] * 32, 32, 1, 6),
    "rows32_two_tokens": (16, _spread(1500, 311, 40), [2] * 40, 32, 0, 30),
    "rows32_long": (28, _spread(8000, 11, 40), [1] * 40, 32, 1, 33),       # more than 16 tiles to each of two waves
    # many rows: the waves have rows of their own
    "rows128": (16, [70, 500], [12, 5], 128, 1, 4),
    "rows128_long": (128, _spread(9800, 13, 64), [1] * 64, 128, 1, 65),    # more than 64 key tiles to a workgroup
    "rows128_even": (16, [0, 3], [2100, 40], 128, 0, 30),
    "rows128_even_long": (16, [2500, 1800], [1100, 1000], 128, 0, 65),     # shares over tiles, more than 64 key tiles of one
}
