"""Rules of order in device code that no result shows reliably, checked in the sources."""
import os
import re

import pytest


def _source(repo_root, name):
    with open(os.path.join(repo_root, "paper_2607_17715_gb300", "csrc", name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _kernel(text, name):
    """The body of kernel `name`."""
    at = text.index("{", text.index(name + "(const __grid_constant__"))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i]


def test_peers_are_written_after_they_have_started(repo_root):
    """Shared memory of a cluster's other CTAs may be accessed only once all of them run: a barrier of the
    cluster lies before the first such store, and its arrival before anything that can return."""
    body = _kernel(_source(repo_root, "verify.cu"), "verify_kernel")
    arrive, wait, store = (body.find(x) for x in ("cluster_started()", "cluster_started_wait()", "st_peer("))
    assert 0 <= arrive < wait < store
    assert "return" not in body[:wait]


OVERLAPPED = ["paged_mma.cu", "paged_lane.cu", "paged_move.cu", "paged_tc.cu", "paged_row.cuh", "verify.cu"]


@pytest.mark.parametrize("name", OVERLAPPED)
def test_overlapped_kernels_load_no_read_only_memory(repo_root, name):
    """A kernel that is set up while the one before it runs waits for it (griddepcontrol.wait) and then loads
    what that wrote: by ordinary loads, since one of memory that never changes may be moved ahead of the wait."""
    text = _source(repo_root, name)
    assert not re.search(r"__ldg\(|\bld16\(|ld\.global(\.\w+)*\.nc", text)
    if name.endswith(".cu"):
        assert "launch_overlapped" in text or "ProgrammaticStreamSerialization" in text
