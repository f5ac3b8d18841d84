"""What the binding of avsg_append and avsg_attend refuses or works out before a call, without a GPU."""
import numpy as np
import pytest

import paper_2609_37538_b200 as avsg
from paper_2609_37538_b200 import binding as b


def test_rows_that_caches_have_room_for():
    import torch
    flat = torch.zeros(10 * 656 + 100, dtype=torch.uint8)
    assert b._rows_in(flat, 656, None) == 10 and b._rows_in(flat, 656, 672) == 9
    assert b._rows_in(flat[::2], 656, None) == 10                       # (its bytes lie within the same range)
    assert b._rows_in(np.zeros(1313, dtype=np.uint8), 656, None) == 2
    assert b._rows_in(np.zeros(100, dtype=np.uint8), 656, None) == 0
    assert b._rows_in(1 << 20, 656, None) is None                       # an address


def test_limits_of_caches():
    assert b._limits([None, None], None) is None
    assert b._limits([None, 7], None) == [0x80000000, 7]
    assert b._limits([None, 7], [100, 7]) == [100, 7]
    for most, rows in (([7, 7], [7, 8]), ([7, 7], [7]), ([None], [1, 2])):
        with pytest.raises(avsg.AvsgError) as e:
            b._limits(most, rows)
        assert e.value.code == avsg.EINVAL


def test_status_words():
    import torch
    word = torch.zeros(2, dtype=torch.int32)
    assert b._status_word(word) == word.data_ptr() and b._status_word(4096) == 4096
    for bad in (torch.zeros(4, dtype=torch.uint8), torch.zeros(1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(avsg.AvsgError):
            b._status_word(bad)


def test_numbers_that_do_not_fit_the_argument_blocks():
    good = [1] * 21
    assert len(b._packed(b._APPEND, "append", *good)) == 152
    for at, wrong in ((0, -1), (0, 1 << 32), (4, "a")):
        values = list(good)
        values[at] = wrong
        with pytest.raises(avsg.AvsgError):
            b._packed(b._APPEND, "append", *values)
