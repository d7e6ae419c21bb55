"""The device headers as they meet in one library.  CPU only."""
import collections
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_14338_b200", "csrc")


def test_no_macro_is_defined_by_two_headers():
    """A kernel template is compiled in every source that uses it, and the library runs any one of these copies.  They
    have to be the same, so no constant may depend on which headers a source includes, or in which order: a macro that
    two headers define, each if the other has not, would size a kernel's shared memory in one source and its
    launch in another."""
    where = collections.defaultdict(set)
    for path in glob.glob(os.path.join(CSRC, "*.cuh")):
        with open(path) as f:
            for name in re.findall(r"^\s*#\s*define\s+(\w+)", f.read(), re.M):
                where[name].add(os.path.basename(path))
    assert where
    assert {n: sorted(p) for n, p in where.items() if len(p) > 1} == {}
