"""What the cache's attention does when a bounded wait has expired, on the host: no copy is left in flight, and a part that came
too late is not taken by the next execution of a captured launch.  CPU only."""
import os
import subprocess

import pytest


@pytest.fixture(scope="module")
def cache_wait(tmp_path_factory, repo_root):
    exe = str(tmp_path_factory.mktemp("wait") / "cache_wait")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-pthread", "-o", exe, os.path.join(repo_root, "tests", "cache_wait.cpp")])
    return exe


@pytest.mark.parametrize("what", ["ring", "replays", "threads"])
def test_expired_waits(cache_wait, what):
    out = subprocess.run([cache_wait, what], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout
