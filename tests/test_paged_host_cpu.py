"""Host code of the paged calls without a GPU, over the stand-in for the CUDA runtime (tests/host)."""
import pytest

from tests.test_host_paths_cpu import _run, program  # noqa: F401


@pytest.mark.parametrize("scenario", ["paged_capture", "paged_no_memory"])
def test_scenario(program, scenario):  # noqa: F811
    _run(program, scenario)
