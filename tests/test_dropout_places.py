"""How dropout's threads find their rows: a place's quotient by the units of a row, as a product's high word (a model of the
kernel's step; no GPU needed)."""
CHUNK = 512  # units that a block takes at a time


def over(at, units):
    if units == 1:
        return at
    if units >= CHUNK:
        return int(at >= units)
    inverse = (2 ** 32 + units - 1) // units
    assert inverse < 2 ** 32
    return at * inverse >> 32


def test_every_place_of_every_row_length():
    for units in range(1, 2 * CHUNK):
        for at in range(units + CHUNK):  # a block's first unit lies in its row, its last CHUNK - 1 behind it
            assert over(at, units) == at // units, (at, units)
