"""Attention calls of one and of two keys under 32-bit queries, whose results say how many bits of a score and of a
probability a kernel keeps, with the bounds of 32-bit arithmetic on them.  Test infrastructure: no code of the library.

One key: its score is one element of the query (the key is one-hot, the scale 1), so lse is that element.  On its way
lie a factor log2 e and a factor ln 2, each rounded itself and rounding its product: 4 * 2^-24 of it, and a spare one.

Two keys of scores 0 and -x, values +1 and -1: out = (1 - e^-x) / (1 + e^-x) = tanh(x / 2), lse = ln(1 + e^-x).  With
x in [1/64, 1/32) e^-x lies in [0.96, 1), where a unit of the last place is 2^-24.  It is off by that unit (the
exponential's) and by what x is, less than 4 * 2^-24 / 32; a factor that joins two parts rounds once more, by half a
unit; the difference from 1 is exact.  Over the sum, 1.96 to 2, that is below 2^-24, and what division and sum add is
below 6 * 2^-24 of an out below 1/64: 2^-23 allows twice that.  lse: 2^-24 for the sum's error over the sum, 2^-24 for
the logarithm's and twice that for the product with ln 2: 2^-22."""
import torch

SCORE = 5 * 2.0 ** -24   # of lse
OUT = 2.0 ** -23
LSE = 2.0 ** -22


def full_mantissas(g, shape, low, high):
    """Values of either sign with magnitudes spread over [low, high), every bit of their significands in use."""
    v = low + (high - low) * torch.rand(shape, generator=g, dtype=torch.float64)
    return (v * (1 - 2 * torch.randint(0, 2, shape, generator=g))).float()


def one_hot(at, n, value=1.0):
    """Rows that are `value` at the places `at` and 0 elsewhere."""
    return torch.nn.functional.one_hot(at, n).float() * value


def expected_of_two(x):
    """(out, lse) of the two keys, x in double."""
    return torch.tanh(x / 2), torch.log1p(torch.exp(-x))
