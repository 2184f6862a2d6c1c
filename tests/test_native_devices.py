"""Calls whose stream is on another device than the current one (tests/native/two_devices.c, built by
tests/native/build_native.py): the scratch and the launches are those of the stream's device. No GPU."""
import os
import subprocess

DRIVER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "_out", "two_devices")


def test_shared_past_on_the_streams_device():
    assert os.path.exists(DRIVER), f"{DRIVER} missing: run tests/native/build_native.py (or __graft_entry__.build())"
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1")
    r = subprocess.run([DRIVER], capture_output=True, text=True, timeout=120, env=env)
    out = r.stdout + r.stderr
    print(out[-4000:])
    assert r.returncode == 0 and "two_devices: ok" in out and "Sanitizer" not in out
