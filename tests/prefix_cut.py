"""The rules by which adsa_shared_prefix_attn cuts its lists of units into runs, restated (numpy, whole arrays at a time)."""
import numpy as np


def _bits(x):
    """Length of x in bits (x >= 0)."""
    return int(x).bit_length()


class Cut:
    """Of the sweep's list: `resident` runs of 2^(K-2) pieces, as many of half that, .. of one piece, and as many of one again."""

    def __init__(self, total, resident):
        self.total, self.resident = total, resident
        fours = min(total // (4 * resident), 16)
        self.K = 1 if fours < 2 else _bits(fours)
        self.half = 1 << (self.K - 1)
        pieces, self.runs = self.half * resident, self.K * resident
        if total < resident:
            pieces = self.runs = max(total, 1)
        self.base, self.rem = total // pieces, total % pieces
        if total == 0:
            self.runs = 0

    def begin_of(self, run):
        run = np.asarray(run, dtype=np.int64)
        p = run
        if self.half > 1:
            k = run // self.resident
            p = (self.half - (self.half >> k)) * self.resident + (run - k * self.resident) * np.maximum(1, self.half >> (k + 1))
            p = np.minimum(p, self.half * self.resident)
        return p * self.base + np.minimum(p, self.rem)

    def run_of(self, unit):
        unit = np.asarray(unit, dtype=np.int64)
        big = self.rem * (self.base + 1)
        p = np.where(unit < big, unit // (self.base + 1), self.rem + (unit - big) // max(self.base, 1))
        if self.half == 1:
            return np.minimum(p, self.runs - 1)
        left = self.half - p // self.resident
        k = (_bits(self.half) - 1) - np.array([_bits(x) for x in range(self.half)])[left - 1]
        return np.minimum(k * self.resident + (p - (self.half - (self.half >> k)) * self.resident) // np.maximum(1, self.half >> (k + 1)),
                          self.runs - 1)


class WideCut:
    """Of the wide kernel's list: even runs of two units or more."""

    def __init__(self, total, resident):
        self.total, self.runs = total, min(resident, total // 2)
        if total > 0 and self.runs == 0:
            self.runs = 1

    def begin_of(self, run):
        return np.asarray(run, dtype=np.int64) * self.total // self.runs

    def run_of(self, unit):
        return ((np.asarray(unit, dtype=np.int64) + 1) * self.runs - 1) // self.total


def sweep_units(own, prefix, start, kv, per, dim, wide_above=1 << 30):
    """Units of the sweep's list."""
    tile = 128 if dim <= 64 else 64
    total = sum(-(-per // 32) * kv * -(-n // tile) for n in own)
    for g, n in enumerate(prefix):
        m = (start[g + 1] - start[g]) * per
        if m <= wide_above:
            total += -(-m // 32) * kv * -(-n // tile)
    return total


def wide_units(prefix, start, kv, per):
    """Units of the wide kernel's list (groups of more than 32 query rows of a key head)."""
    total = 0
    for g, n in enumerate(prefix):
        m = (start[g + 1] - start[g]) * per
        if m > 32:
            total += -(-m // 128) * -(-n // 128) * kv
    return total
