"""Recorded steps of pools in 8 bits: one is updated in place only from one of the same kernels (compiled with gcc under
AddressSanitizer + UndefinedBehaviorSanitizer, tests/hostbuild/kv8_recordings_main.cpp).  No GPU."""
import os

from test_host_kv8 import HB, _build, _run


def test_a_recording_is_updated_from_one_of_the_same_kernels(tmp_path):
    exe = str(tmp_path / "kv8_recordings")
    _build(exe, [os.path.join(HB, "kv8_recordings_main.cpp")])
    _run(exe)
