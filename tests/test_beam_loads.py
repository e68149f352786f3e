"""How the beam search's and the shared pages' kernels read global memory, from their sources (CPU only)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_14898_gb300", "csrc")


@pytest.mark.parametrize("name", ["beam.cu", "kv_pages.cu"])
def test_nothing_is_read_as_if_it_never_changed(name):
    """A kernel is launched while the one before it still runs, and may be writing what this one reads behind its wait: the loads that
    take memory for read-only as long as the kernel lives are none for it."""
    with open(os.path.join(CSRC, name)) as fh:
        code = "\n".join(line.split("//", 1)[0] for line in fh)
    assert not re.search(r"__ldg\s*\(|\.nc\b|__restrict__", code)
