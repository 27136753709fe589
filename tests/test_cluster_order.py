"""Another block's shared memory may be accessed only once that block is known to run: in the text of every kernel that maps an
address into one, a cluster-wide wait stands before the first such address.  Read from the sources: a race on memory is not
something to be provoked."""
import glob
import os
import re

import pytest

from paper_1910_11971_gb300 import build as cci_build

WAIT = re.compile(r"cluster_sync\(\)|cluster\.sync\(\)|barrier_wait\(\)|barrier\.cluster\.wait")
REMOTE = re.compile(r"map_to_rank\(|map_shared_rank\(")


def kernels():
    """(file and name, text) of each kernel that maps an address into another block."""
    found = []
    for path in sorted(glob.glob(os.path.join(cci_build.CSRC, "*.cu*"))):
        with open(path) as f:
            text = f.read()
        for part in re.split(r"(?m)^__global__", text)[1:]:
            body = part[:part.index("\n}\n")]  # ends with the kernel's own brace
            if REMOTE.search(body):
                name = re.search(r"\b(\w*kernel\w*)\(", body).group(1)
                found.append((f"{os.path.basename(path)}: {name}", body))
    return found


KERNELS = kernels()


def test_there_are_such_kernels():
    assert len(KERNELS) >= 7, [name for name, _ in KERNELS]


@pytest.mark.parametrize("name,body", KERNELS, ids=[name for name, _ in KERNELS])
def test_a_wait_stands_before_the_first_access(name, body):
    first, wait = REMOTE.search(body), WAIT.search(body)
    assert wait is not None and wait.start() < first.start()
