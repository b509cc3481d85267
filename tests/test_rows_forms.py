"""Every kernel of the operators on rows of scores that is compiled has calls
that run it."""
import re
import shutil
import subprocess

import pytest

import paper_2508_07315_amd as P
import rows_calls
from rows_forms import Forms


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    return Forms(tmp_path_factory.mktemp("forms"))


def compiled():
    """The kernels in the library, by the names of their launch functions."""
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("needs nm")
    P._load()
    text = subprocess.run([nm, "-C", P.library_path()], capture_output=True, text=True, check=True).stdout
    found = re.findall(r"ctcbeam::rows::__device_stub__((?:process|top|distill|join)\w*(?:<[^>]*>)?)\(", text)
    return {f.replace("ctcbeam::rows::", "") for f in found}


def test_compiled_and_reachable_kernels_are_the_same(forms):
    have, reached = compiled(), forms.all()
    assert reached - have == set(), "plans that pick a kernel which is not compiled"
    assert have - reached == set(), "kernels that no call runs"


def test_every_kernel_is_run_on_the_gpu(forms):
    calls = list(rows_calls.every())
    run = {f for found in forms.of(calls) for f in found}
    assert forms.all() - run == set()
    assert {"counts for several frames, 64", "counts for several frames, 256"} <= run
