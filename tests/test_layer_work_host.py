"""The work memory of the operators of a sparse layer, without a GPU (see layer_work_calls.py): one process per case."""
import subprocess
import sys

import pytest

from tests import host_calls


@pytest.fixture(scope="module", autouse=True)
def stub():
    host_calls.build()


@pytest.mark.parametrize("case", ["bounds", "too_little", "groups"])
def test_host_code(case):
    r = subprocess.run([sys.executable, "-m", "tests.layer_work_calls", case], cwd=host_calls.ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout + r.stderr
