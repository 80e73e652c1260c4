"""What the kernels' sources may not contain.

libmtsim is loaded by every rank of a run on several GPUs, and its entry points
take any address.  A copy that one block makes into several blocks' shared
memory is only for memory of the block's own GPU, so no kernel of the library
has one."""
import os

from paper_2608_16336_gb300 import _build


def test_no_copy_goes_to_several_blocks():
    sources = [p for p in _build.mtsim_sources() if p.startswith(_build.CSRC)]
    assert sources
    for path in sources:
        assert "multicast" not in open(path).read(), os.path.basename(path)
