"""Workspace queries answer for what the calls take and refuse the rest, without a GPU."""
import os
import subprocess
import sys

from tests.test_operator_calls import HOST, LIB, fake, pytestmark  # noqa: F401


def test_queries_on_a_runtime_that_only_books(fake):  # noqa: F811
    res = subprocess.run([sys.executable, os.path.join(HOST, "operator_workspaces.py"), fake, LIB],
                         capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "passed" in res.stdout, res.stdout + res.stderr
