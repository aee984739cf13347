"""What the package's small language model refuses, and what it reports."""
import subprocess
import sys

import pytest

import paper_2205_14473_gb300 as ea
from paper_2205_14473_gb300 import bigram


def test_dropout_needs_blocks(ea_lib):
    with pytest.raises(ValueError, match="blocks"):
        bigram.Bigram(16, 8, 16, "cuda", dropout=0.1)
    r = subprocess.run([sys.executable, "-m", bigram.__name__, "--dropout", "0.1"], capture_output=True, text=True)
    assert r.returncode == 2 and "--blocks" in r.stderr


@pytest.mark.gpu
def test_training_reports_the_status_of_the_recurrence(monkeypatch):
    """A wait within a cluster that ran out (here: that is said to have) does not pass as a result."""
    import __graft_entry__

    __graft_entry__.build()

    def sync(scan):
        raise ea.EAError(ea.EA_E_TIMEOUT, "a wait ran out")

    monkeypatch.setattr(ea.GatedScan, "sync", sync)
    assert len(bigram.train(steps=1, workers=1)) == 1
    with pytest.raises(ea.EAError) as ex:
        bigram.train(steps=1, workers=1, blocks=1)
    assert ex.value.status == ea.EA_E_TIMEOUT
