"""Stores of 16 bytes have no scalar register as an offset: with one, the compiler lets the next vector instruction write the data's registers
while the store still reads them.  Read from the sources; no GPU."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_10639_amd", "csrc")
CALL = re.compile(r"raw_(?:ptr_)?buffer_store_(?:b96|b128)\s*\(")


def arguments(text, at):
    depth, start, out = 0, at, []
    for i in range(at, len(text)):
        if text[i] in "([{":
            depth += 1
        elif text[i] in ")]}":
            if depth == 0:
                return out + [text[start:i].strip()]
            depth -= 1
        elif text[i] == "," and depth == 0:
            out.append(text[start:i].strip())
            start = i + 1


@pytest.mark.parametrize("path", sorted(glob.glob(CSRC + "/*.hip") + glob.glob(CSRC + "/*.h")), ids=os.path.basename)
def test_scalar_offsets_of_wide_stores_are_constants(path):
    text = open(path).read()
    for call in CALL.finditer(text):
        args = arguments(text, call.end())
        # (a constant that an instruction holds by itself: 0 to 64)
        assert len(args) == 5 and args[3].isdigit() and int(args[3]) <= 64, (text.count("\n", 0, call.start()) + 1, args)
