"""The generator behind the dropout's reference, against published vectors of Philox4x32-10 (CPU)."""
import numpy as np
import pytest

from residual_cases import kept, philox, threshold

VECTORS = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


@pytest.mark.parametrize("counter,key,want", VECTORS)
def test_published_vectors(counter, key, want):
    assert tuple(int(w) for w in philox(counter, key)) == want


def test_the_kept_share():
    n, C = 4000, 80
    for p in (0.0, 0.1, 0.5, 0.9, 1.0):
        share = float(kept((7, 3), n, C, p).double().mean())
        q = threshold(p) / 65536
        assert abs(share - (1 - q)) <= 6 * np.sqrt(q * (1 - q) / (n * C))
    assert threshold(1e-6) == 0 and threshold(0.5) == 32768 and threshold(1.0) == 65536


def test_calls_seeds_rows_and_channels_have_bits_of_their_own():
    a = kept((7, 3), 50, 20, 0.5)
    for other in (kept((8, 3), 50, 20, 0.5), kept((7, 4), 50, 20, 0.5), kept((7 + 2 ** 32, 3), 50, 20, 0.5), kept((7, 3 + 2 ** 32), 50, 20, 0.5)):
        assert 0.35 < float((a != other).double().mean()) < 0.65
    assert (kept((7, 3), 50, 20, 0.5)[:, :17] == kept((7, 3), 60, 17, 0.5)[:50]).all()      # whatever the shape
