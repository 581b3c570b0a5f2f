"""Every bounded wait on the device leaves a code of its own in the status word, by which a wait that ran out is found."""
import collections
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_13645_b200", "csrc")


def test_no_two_waits_share_a_code():
    at = collections.defaultdict(list)
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        for n, line in enumerate(open(path), 1):
            if re.search(r"\b(mbar_wait|wait_all)\(", line):
                for code in re.findall(r"\b0x[0-9a-f]{2}\b(?=\)| \|)", line):
                    at[code].append(f"{os.path.basename(path)}:{n}")
    assert len(at) >= 60
    assert not {c: where for c, where in at.items() if len(where) > 1}
