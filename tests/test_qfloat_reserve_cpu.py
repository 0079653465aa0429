"""The 8-bit floating point calls' scratch where memory ends half-way: nothing is left over that a later call would take for its own."""
import ctypes
import itertools

import pytest

from paper_2601_10639_amd import stemlib as L


class Room(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int), ("backward", ctypes.c_int), ("p", ctypes.c_void_p * 5)]


TAKE = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int64)
GIVE = ctypes.CFUNCTYPE(None, ctypes.c_void_p)
T, WIDE, F = 1000, 320, 192


class Memory:
    """Buffers by address; the call number `ends` and those behind it get none."""

    def __init__(self):
        self.held, self.next, self.left = {}, itertools.count(0x10000, 0x1000), None

    def call(self, room, groups, backward, left=None):
        self.left = left

        def take(at, size):
            if self.left is not None:
                if self.left == 0:
                    return 2
                self.left -= 1
            at[0] = address = next(self.next)
            self.held[address] = size
            return 0

        def give(address):
            del self.held[address]

        f = L.lib().stem_qfloat_room_take
        f.argtypes = [ctypes.POINTER(Room), ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int, TAKE, GIVE]
        return f(ctypes.byref(room), T, WIDE, F, groups, backward, TAKE(take), GIVE(give))


def sizes(groups, backward):
    rows, pad = 1024 + 128 * (min(groups, T) - 1), lambda n: -(-n // 128) * 128
    form = lambda k: rows * pad(k) // 128 * 129
    return [form(WIDE), form(F), 256 * 128 * 128 * 4] + ([2 * rows * pad(WIDE)] * 2 if backward else [])


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("left", range(5))
def test_the_first_call_fails(left, backward):
    if left >= (5 if backward else 3):
        pytest.skip("it does not fail then")
    m, room = Memory(), Room()
    assert m.call(room, 2, backward, left) == 2
    assert room.groups == 0 and room.backward == 0 and not any(room.p) and not m.held
    assert m.call(room, 100, backward) == 0                               # names more
    assert room.groups == 100 and room.backward == backward
    assert [m.held[p] for p in room.p if p] == sizes(100, backward) and len(m.held) == 3 + 2 * backward


@pytest.mark.parametrize("left", [0, 1])
def test_the_backward_pass_is_added_later(left):
    m, room = Memory(), Room()
    assert m.call(room, 7, 0) == 0
    before, held = list(room.p), dict(m.held)
    assert m.call(room, 3, 1, left) == 2
    assert list(room.p) == before and m.held == held and (room.groups, room.backward) == (7, 0)
    assert m.call(room, 3, 1) == 0
    assert list(room.p)[:3] == before[:3] and [m.held[p] for p in room.p] == sizes(7, 1) and (room.groups, room.backward) == (7, 1)
    assert m.call(room, 7, 1, 0) == 0 and m.call(room, 1, 0, 0) == 0      # all there already
    assert len(m.held) == 5
