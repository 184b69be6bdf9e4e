"""The compiled norms, rotary embedding and vocabulary head hold no result read too early and no copy under a
partial mask (wait_states.py)."""
import os
import subprocess

import pytest
import wait_states as W

from paper_2502_19864_amd import build


@pytest.mark.parametrize("source,least", [("k_norm.hip", 45), ("k_rotary.hip", 4), ("k_vocab.hip", 18), ("k_vocab_mm.hip", 20)])
def test_compiled_kernels(source, least, tmp_path):
    out = str(tmp_path / "k.s")
    subprocess.run([build.hipcc()] + build.flags() + ["-S", "--cuda-device-only", os.path.join(build.CSRC, source),
                                                     "-o", out], check=True, capture_output=True)
    n = 0
    for name, ins, labels in W.kernels(open(out).read()):
        n += 1
        assert not W.short_waits(ins, labels), name
        assert not W.masked_copies(ins, labels), name
    assert n >= least
