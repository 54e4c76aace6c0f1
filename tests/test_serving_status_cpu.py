"""Attention calls that give up a bounded wait are heard of: every wait of their kernels names the device's status word, and
the call that reads it never says that all is well where it cannot be read."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_37924_gb300", "csrc")


@pytest.mark.parametrize("name", ["attention_packed.cu", "attention_paged.cu"])
def test_every_bounded_wait_names_the_status_word(name):
    src = open(os.path.join(CSRC, name)).read()
    waits = re.findall(r"(?:mbar|warp)_wait_bounded\((.*)\)", src)
    assert len(waits) > 8
    for w in waits:
        assert "a.status" in w and "nullptr" not in w, w


def test_status_without_a_device():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    import __graft_entry__ as g
    g.build()
    from paper_2609_37924_gb300 import tadm
    assert tadm.load_library().tadm_ragged_sync_status(None) == 3          # TADM_ERR_CUDA


def test_the_wrapper_raises(monkeypatch):
    from paper_2609_37924_gb300 import tadm

    class Library:
        tadm_ragged_sync_status = staticmethod(lambda stream: 5)           # TADM_ERR_TIMEOUT

    monkeypatch.setattr(tadm, "load_library", lambda *a: Library)
    monkeypatch.setattr(tadm, "_stream", lambda stream=None: None)
    with pytest.raises(tadm.TadmError) as e:
        tadm.tadm_ragged_sync_status()
    assert e.value.status == 5
