"""Tests of files named test_zz_* run behind all others, in whatever order files are asked for."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_what_has_to_run_last_does():
    """Streams share a few hardware queues, and test_zz_streams_of_ends.py puts two more to use: a test that copies to the host beside a daemon that does not leave by itself
    may then wait for that daemon, and runs before."""
    files = ["test_zz_streams_of_ends.py", "test_gpu_scheduling.py", "test_zz_no_alloc.py", "test_tiles.py"]
    out = subprocess.run([sys.executable, "-m", "pytest", "--collect-only", "-q", "-p", "no:cacheprovider"] + [os.path.join("tests", f) for f in files], cwd=ROOT, capture_output=True, text=True,
                         timeout=300)
    order = list(dict.fromkeys(os.path.basename(line.split("::")[0]) for line in out.stdout.splitlines() if "::" in line))
    assert order == ["test_gpu_scheduling.py", "test_tiles.py", "test_zz_no_alloc.py", "test_zz_streams_of_ends.py"], out.stdout[-2000:] + out.stderr[-2000:]
