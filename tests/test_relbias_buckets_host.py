"""The kernels' lookups of buckets and of their starts stay inside the array that holds the starts, for every number of buckets that the library accepts:
their header built as plain C++ with the bounds of arrays checked (tests/relbias_buckets_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which(os.environ.get("CXX", "g++")) is None, reason="no host C++ compiler")
def test_lookups_stay_inside_the_starts(tmp_path):
    exe = str(tmp_path / "relbias_buckets")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-g", "-Wall", "-Wno-unknown-pragmas", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    os.path.join(HERE, "relbias_buckets_driver.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "relative bias buckets: ok" in r.stdout and "runtime error" not in r.stderr, (r.stdout[-2000:], r.stderr[-2000:])
