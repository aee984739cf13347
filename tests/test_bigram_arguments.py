"""What the package's small language model refuses, and what it reports."""
import subprocess
import sys

import pytest

from paper_2205_14473_gb300 import bigram


def test_dropout_needs_blocks(ea_lib):
    with pytest.raises(ValueError, match="blocks"):
        bigram.Bigram(16, 8, 16, "cuda", dropout=0.1)
    r = subprocess.run([sys.executable, "-m", bigram.__name__, "--dropout", "0.1"], capture_output=True, text=True)
    assert r.returncode == 2 and "--blocks" in r.stderr
