"""As test_lds_waits, for the 8-bit layer's kernels; and the loads that go straight into LDS: a wavefront waits for its own
before the barrier behind which others read them."""
import os
import re
import subprocess

import pytest

from paper_2506_16235_amd import build as B
from test_lds_waits import _unfinished


@pytest.mark.parametrize("unit", B.LAYER8_UNITS)
def test_no_lds_write_in_flight_at_a_barrier(unit, tmp_path):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path / "k.s")
    flags = [f for f in B.HIP_FLAGS if f != "-fPIC"]
    subprocess.run([B.HIPCC, *flags, "-I", B.INCLUDE, "--cuda-device-only", "-S", os.path.join(B.LAYER8, unit + ".hip"), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    assert text.count("s_barrier") >= 3
    assert _unfinished(text) == []
    assert not re.search(r"v_pk_(add|mul|fma)_f32", text)
