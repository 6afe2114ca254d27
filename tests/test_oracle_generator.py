"""The dropout's generator against the published answers of Philox4x32-10 for every key and counter word (no GPU)."""

import numpy as np
import pytest

from oracle import ends as OE


def philox4x32(counter, key):
    """Ten rounds on four counter words and two key words (Salmon et al., SC 2011), on plain integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b % 2 ** 32, (a >> 32) ^ c[3] ^ k[1], a % 2 ** 32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


@pytest.mark.parametrize("counter,key,words", [
    ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])])
def test_published_answers(counter, key, words):
    assert philox4x32(counter, key) == words


@pytest.mark.parametrize("key", [0, 1, 1 << 32, 0x299F31D0A4093822, 2 ** 64 - 1, 12345678901234567890])
@pytest.mark.parametrize("counter", [0, 1, 2 ** 32 - 1, 2 ** 32, 0x85A308D3243F6A88, 2 ** 64 - 1])
def test_oracle_draws_the_published_words(key, counter):
    # the key's and the counter's low words come first; the counter's upper 64 bits are zero
    want = philox4x32([counter % 2 ** 32, counter >> 32, 0, 0], [key % 2 ** 32, key >> 32])
    assert OE.philox(key, counter, 1)[0].tolist() == want
    assert np.array_equal(OE.dropout_keep(4, 0.5, key, counter), [w >= 2 ** 31 for w in want])
