"""What keeps the calls with several new tokens per sequence from touching what is not theirs, on
the CPU: everything here ends before a launch."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def hk():
    import paper_2606_28831_amd as hk
    return hk


I32 = torch.int32


def test_the_word_of_granted_chunks(hk):
    """Chunks carry their decoder's word to later calls; anything but an int32 word of the starts'
    device is refused."""
    start, word = torch.zeros(3, dtype=I32), torch.ones(1, dtype=I32)
    ch = hk.Chunks(start, 4, 4)
    assert ch.granted is None and ch.desc.granted is None
    ch = hk.Chunks(start, 4, 4, granted=word)
    assert ch.desc.granted == word.data_ptr() and C.sizeof(ch.desc) == 32
    ch.granted_by(None)
    assert ch.desc.granted is None
    for bad in (torch.ones(1), torch.ones(1, dtype=torch.int64), torch.zeros(0, dtype=I32), torch.empty(1, dtype=I32, device="meta")):
        with pytest.raises(hk.HardKVError):
            ch.granted_by(bad)
    assert ch.granted is None
