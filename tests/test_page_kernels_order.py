"""What the page operators' kernels promise to the attention kernels, which read tables and lengths before they wait for the kernel
before them, read in the sources (when a kernel starts cannot be set from a test)."""
import pytest

from tests.test_cluster_stores import kernels

BODIES = dict(kernels("pages.cu"))


def test_the_copy_signals_only_behind_its_wait():
    body = BODIES["copy_pages_kernel"]
    assert 0 <= body.find("grid_dependency_wait()") < body.find("grid_dependency_launch()")


@pytest.mark.parametrize("name", ["fork_share_kernel", "compact_move_kernel"])
def test_a_calls_last_kernel_that_writes_tables_never_signals(name):
    assert "grid_dependency_wait()" in BODIES[name] and "grid_dependency_launch()" not in BODIES[name]


def test_the_last_kernel_of_a_resize_never_signals():
    """(One kernel for copies alone and behind a resize, by its template argument.)"""
    lines = [line for line in BODIES["copy_pages_kernel"].splitlines() if "grid_dependency_launch()" in line]
    assert len(lines) == 1 and lines[0].strip().startswith("if (!kRows) ")
