"""The generator that the device's dropout is compared with, against its authors' test vectors."""
import pytest

from test_gpu_language import _pieces

ONES = 0xFFFFFFFF


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((ONES,) * 4, (ONES,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_pieces_have_the_published_words(counter, key, want):
    """Philox-4x32-10: the counter's words are the block's two and the offset's two, the key's the
    seed's, low ones first. The last vector's six words differ from each other."""
    block, offset = counter[0] | counter[1] << 32, counter[2] | counter[3] << 32
    p = _pieces(8, key[0] | key[1] << 32, offset, first=8 * block)
    assert tuple(int(p[2 * i] | p[2 * i + 1] << 16) for i in range(4)) == want
