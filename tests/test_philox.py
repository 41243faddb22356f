"""The restated generator against the known answers published with it, and the shares it drops."""
import numpy as np
import pytest

from philox import kept, numbers, philox4x32


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_known_answers(counter, key, want):
    got = philox4x32([np.array([v]) for v in counter], key)
    assert tuple(int(v[0]) for v in got) == want


def test_numbers_of_a_range_are_those_of_the_whole():
    whole = numbers(0, 1000, 5, 6)
    assert (numbers(123, 500, 5, 6) == whole[123:623]).all()
    assert whole.max() < 65536
    assert not kept((1000,), 1.0, 5, 6).any() and kept((1000,), 0.0, 5, 6).all()
    n = 200_000
    share = 1 - kept((n,), 0.3, 9, 2 ** 40).double().mean().item()
    assert abs(share - 0.3) < 5 * (0.3 * 0.7 / n) ** 0.5
