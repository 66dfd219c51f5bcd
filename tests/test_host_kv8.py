"""Host paths of pools in 8 bits (block tables cut into launches, read-back lists, step forms, the rotating append) compiled
with gcc under AddressSanitizer + UndefinedBehaviorSanitizer, with stand-ins for the launchers that check every row of
every launch (tests/hostbuild/kv8_main.cpp); and a build without the 8-bit kernels, which refuses.  No GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HB = os.path.join(ROOT, "tests", "hostbuild")
CSRC = os.path.join(ROOT, "paper_2603_14371_amd", "csrc")


def _build(target, sources):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-fno-omit-frame-pointer", "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           os.path.join(CSRC, "oxy_pool.cpp"), os.path.join(CSRC, "oxy_sched.cpp"), os.path.join(HB, "hip_stubs.cpp")]
    res = subprocess.run(cmd + sources + ["-o", target], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]


def _run(exe):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert res.returncode == 0 and res.stdout.startswith("OK"), res.stdout[-4000:]


def test_every_row_of_every_launch(tmp_path):
    exe = str(tmp_path / "kv8_asan")
    _build(exe, [os.path.join(HB, "kv8_main.cpp")])
    _run(exe)


def test_a_build_without_the_kernels_refuses(tmp_path):
    src = tmp_path / "without.cpp"
    src.write_text("""
#include "%s/include/oxy.h"
#include <cstdio>
#include <cstdlib>
#include <cstring>
int main() {
  oxy_pool_config c;
  memset(&c, 0, sizeof(c));
  c.n_layers = 1, c.n_q_heads = 8, c.n_kv_heads = 1, c.head_dim = 256, c.page_size = 16, c.num_blocks = 4;
  c.max_q_tokens = c.max_append_tokens = 16;
  c.kv_base = c.workspace = aligned_alloc(256, 64 << 20);
  c.kv_bytes = c.workspace_bytes = 64 << 20;
  oxy_pool *p = nullptr, *q = nullptr;
  if (oxy_pool_create(&c, &p) != OXY_OK) return 1;
  int32_t sid = 0;
  oxy_batch* b = nullptr;
  oxy_stream_create(p, -1, OXY_KIND_DECODE, &sid);
  oxy_item it = {sid, 2};
  if (oxy_batch_build(p, &it, 1, 0, nullptr, &b) != OXY_OK) return 2;
  double f = 1.0;
  oxy_rotary_config r = {2, 0, &f, 1.0};
  if (oxy_rotary_append(p, b, 0, &r, &sid, nullptr, 0, nullptr, c.kv_base, 512, c.kv_base, 512, nullptr) != OXY_ERR_INVALID_ARG)
    return 3;
  oxy_batch_destroy(b);
  oxy_pool_destroy(p);
  c.flags = OXY_POOL_KV_FP8;
  if (oxy_pool_create(&c, &q) != OXY_ERR_INVALID_ARG || q) return 4;
  free(c.kv_base);
  printf("OK\\n");
  return 0;
}
""" % ROOT)
    exe = str(tmp_path / "without")
    _build(exe, [str(src)])
    _run(exe)
