"""CPU-only: every tensor map has the form that its encoder documents, in which a stride includes the dimensions before it.  One of
two dimensions has it by its leading dimension; maps of more dimensions over matrices that lie anywhere would not."""
import glob
import os
import re

from paper_2504_06323_b200 import build

CSRC = os.path.join(os.path.dirname(build.__file__), "csrc")


def test_maps_are_of_one_matrix_in_two_dimensions():
    ranks, loads = [], []
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        with open(path) as f:
            text = f.read()
        ranks += re.findall(r"\bencode\(map, [^,]+, (\d)u", text)
        loads += re.findall(r"cp\.async\.bulk\.tensor\.(\d)d", text)
    assert len(ranks) >= 2 and set(ranks) == {"2"}
    assert len(loads) >= 2 and set(loads) == {"2"}
