"""The gradients of the selective scan put a step's sums where the step's row stood: the lanes of a channel, which all read that row, have to have done
so by then.  A shuffle in between orders no accesses to shared memory, and which lane gets there first cannot be forced in a run, so the order
is looked up in the source."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_lanes_wait_for_one_another_before_sums_replace_a_row():
    with open(os.path.join(ROOT, "paper_2509_16434_b200", "csrc", "selective_scan.cu")) as f:
        text = f.read()
    body = text[text.index("scan_bwd_kernel("):text.index("scan_few_kernel(")]
    stores = [m.start() for m in re.finditer(r"&s\.su\[r\]\[local\] : &s\.sg\[r\]\[local - 4\]\) \+ at\) = ", body)]
    assert len(stores) == 1
    reads = max(body.rindex(f"load_pairs(&s.{row}[r][local]", 0, stores[0]) for row in ("su", "sg"))
    assert "__syncwarp();" in body[reads:stores[0]]
