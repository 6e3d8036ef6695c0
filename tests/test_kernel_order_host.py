"""Kernels are launched as programmatic dependents of what precedes them in their stream, so that nothing but their own wait orders what they read and write behind
it.  Read from the sources: each kernel waits, whatever its arguments are, and no block leaves without."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2211_10482_b200", "csrc")


def matching(text, at, pair="{}"):
    """The place behind the bracket that closes the one at `at`."""
    depth = 0
    for i in range(at, len(text)):
        depth += (text[i] == pair[0]) - (text[i] == pair[1])
        if depth == 0:
            return i + 1
    raise AssertionError("a bracket that is not closed")


def kernels():
    """(file, name, body) of every kernel but those that are launched without the attribute, by <<< >>>."""
    found, plain = [], set()
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"/\*.*?\*/", "", re.sub(r"//[^\n]*", "", f.read()), flags=re.S)
        plain.update(re.findall(r"\b(\w+)\s*<<<", text))
        for m in re.finditer(r"\b__global__\b", text):
            at = m.end()
            bounds = re.match(r"[\s\w]*__launch_bounds__\s*", text[at:])
            if bounds:
                at = matching(text, at + bounds.end(), "()")
            called = re.match(r"\s*(?:void\s+)?(\w+)\s*(?=\()", text[at:])
            args = matching(text, at + called.end(), "()")
            assert text[args:].lstrip()[0] == "{", (name, called.group(1))
            body = text.index("{", args)
            found.append((name, called.group(1), text[body : matching(text, body)]))
    return [k for k in found if k[1] not in plain]


KERNELS = kernels()


def test_the_kernels_are_found():
    assert len(KERNELS) >= 30 and {"cells_step_kernel", "shared_prefix_kernel", "rotate_kernel", "window_kernel"} <= {k for _, k, _ in KERNELS}


@pytest.mark.parametrize("name,kernel,body", KERNELS, ids=["%s:%s" % k[:2] for k in KERNELS])
def test_each_kernel_waits_for_those_before_it(name, kernel, body):
    waits = [m.start() for m in re.finditer(r"\bpdl_wait\(\)", body)]
    assert waits, "no wait at all"
    first = body[1 : waits[0]]
    while True:                                            # what is in a block that is closed again
        less = re.sub(r"\{[^{}]*\}", ";", first)
        if less == first:
            break
        first = less
    # a statement of the function itself: in no block, behind no condition, and no way out ahead of it
    assert "{" not in first, "within a block"
    assert re.search(r"(^|;)\s*$", first), "behind a condition: %r" % first[-60:]
    assert not re.search(r"\breturn\b", first), "a way out ahead of it"
