"""Accesses through buffer descriptors: the hardware compares a lane's own offset with the buffer's size, and
leaves out the offset that all lanes share.  A kernel that relies on the comparison has to have the whole
place in the lane's offset.  Nothing that a call returns shows it where a kernel does not: what was
read from behind the rows belongs to outputs that are not stored.  So the sources are looked at."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_04702_amd", "csrc")
CALL = re.compile(r"__builtin_amdgcn_raw_(?:ptr_)?buffer_(load_lds|load|store|atomic)\w*\s*\(")
SHARED = {"load": 2, "store": 3, "atomic": 3, "load_lds": 4}  # which argument is the offset that all lanes share


def arguments(text, at):
    """The arguments of a call whose bracket opens just before `at`."""
    depth, args, start = 1, [], at
    for i in range(at, len(text)):
        c = text[i]
        if c in "([{":
            depth += 1
        elif c in ")]}":
            depth -= 1
        if (c == "," and depth == 1) or depth == 0:
            args.append(text[start:i].strip())
            start = i + 1
        if depth == 0:
            return args
    raise AssertionError("a call that does not end")


def calls():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        with open(path) as f:
            text = f.read()
        for m in CALL.finditer(text):
            yield os.path.basename(path), text.count("\n", 0, m.start()) + 1, m.group(1), arguments(text, m.end())


def test_there_are_such_calls():
    assert {kind for _, _, kind, _ in calls()} >= {"load", "store", "load_lds"}


@pytest.mark.parametrize("path,line,kind,args", [pytest.param(*c, id=f"{c[0]}:{c[1]}") for c in calls()])
def test_the_whole_place_is_compared(path, line, kind, args):
    assert args[SHARED[kind]] == "0", f"{path}:{line}: {args}"
