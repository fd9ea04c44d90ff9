"""Calls of several host threads on one stream, which share a library-owned workspace
(or the one that is set): each call's kernels are enqueued together, and a release
does not come between (no GPU; the library's host code with stand-ins for the HIP
runtime and the launchers).  Under ThreadSanitizer where it is installed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "sanitize")


@pytest.mark.parametrize("sanitizer", ["", "thread"])
def test_calls_of_several_threads(tmp_path, sanitizer):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "threads")
    flags = ["-fsanitize=" + sanitizer] if sanitizer else []
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-Wall", *flags, "-I", os.path.join(HERE, "host"), "-I",
                        os.path.join(ROOT, "include"), os.path.join(HERE, "threads_driver.cpp"), "-o", exe, "-lpthread"],
                       capture_output=True, text=True)
    if sanitizer and r.returncode != 0 and "cannot find" in r.stderr:
        pytest.skip("sanitizer runtime not installed")
    assert r.returncode == 0, r.stderr
    env = dict(os.environ)
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    if sanitizer and "unexpected memory mapping" in r.stderr:   # the sanitizer cannot run on this kernel
        pytest.skip("sanitizer does not run here")
    assert r.returncode == 0, r.stdout + r.stderr
    assert "0 refused, 0 met" in r.stdout
