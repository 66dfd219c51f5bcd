"""Host paths of a prefill compiled with gcc under AddressSanitizer + UndefinedBehaviorSanitizer, with a stand-in for the
launch that takes its work list apart (tests/hostbuild/prefill_main.cpp).  No GPU."""
import os

from test_host_kv8 import HB, _build, _run


def test_every_pair_of_every_work_list(tmp_path):
    exe = str(tmp_path / "prefill_asan")
    _build(exe, [os.path.join(HB, "prefill_main.cpp")])
    _run(exe)
