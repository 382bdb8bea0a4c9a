"""A fence orders the initialisations of the thread that executes it and no other's: the thread that initialises a
barrier for the copy engine is the one that fences, in the same branch, behind the last of them.  Read from the sources."""
import os
import re

import pytest

from .plans import CSRC

FILES = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def enclosing_block(text, at):
    """(head, body) of the innermost braces around `at` whose statement is an `if`."""
    depth = 0
    for i in range(at, -1, -1):
        depth += (text[i] == "}") - (text[i] == "{")
        if depth < 0:
            depth = 0
            head = text[text.rfind("\n", 0, i) + 1:i]
            if not re.match(r"\s*if\b", head):
                continue
            end, n = i, 0
            while True:
                n += (text[end] == "{") - (text[end] == "}")
                if n == 0:
                    return head.strip(), text[i:end + 1]
                end += 1
    return "", ""


@pytest.mark.parametrize("name", FILES)
def test_one_thread_initialises_and_fences(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    for m in re.finditer(r"\bmbar_init\(", text):
        head, body = enclosing_block(text, m.start())
        assert re.fullmatch(r"if \((tid|lane|threadIdx\.x) == 0\)", head), (name, text[m.start():m.start() + 80])
        assert body.rfind("fence_barrier_init()") > body.rfind("mbar_init("), (name, head)


def test_some_barriers_are_found():
    n = sum(len(re.findall(r"\bmbar_init\(", open(os.path.join(CSRC, f)).read())) for f in FILES)
    assert n >= 2
