"""The kernels that share one tiled product (monarch_nt.h) read LDS by assembly too: no register of a read in flight is touched before its wait."""
import os
import subprocess

import pytest

from paper_2204_00595_amd import build
from test_lds_reads_in_flight import touched_in_flight


@pytest.mark.parametrize("source", ["monarch_xent.hip", "monarch_ortho.hip"])
def test_no_register_of_a_read_in_flight_is_touched(source, tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path / "device.s"
    subprocess.check_call([build.HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", "-o", str(out), os.path.join(build.CSRC, source)],
                          stderr=subprocess.DEVNULL)
    reads, bad = touched_in_flight(out.read_text().splitlines())
    assert reads > 0 and not bad, (reads, bad[:5])
