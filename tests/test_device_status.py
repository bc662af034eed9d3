"""What a report of vbq_device_status costs: every status word that it reads is a copy that waits for the device."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02893_gb300", "csrc")


def test_four_words_are_read():
    """The products' two, the cache's and its attention's; whatever else reports does so into one of these."""
    reads = {}
    for f in glob.glob(os.path.join(CSRC, "*.cu*")):
        n = len(re.findall(r"cudaMemcpyFromSymbol", open(f).read()))
        if n:
            reads[os.path.basename(f)] = n
    assert reads == {"vbq_gemv.cu": 1, "vbq_gemm.cu": 1, "vbq_kv.cu": 1, "vbq_attend.cu": 1}
