"""The committed traffic figures carry a hash of the sources they were measured on: all that the measured kernels are
compiled from.  No GPU."""
import json
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2603_14371_amd", "csrc")


def includes(name, seen):
    seen.add(name)
    for inner in re.findall(r'#include "([^"]+)"', open(os.path.join(CSRC, name)).read()):
        if inner not in seen:
            includes(inner, seen)
    return seen


def test_every_source_of_the_kernels_is_hashed():
    assert sorted(includes("oxy_kernels.hip", set())) == sorted(bench.KERNEL_SOURCES)


def test_a_change_of_any_of_them_changes_the_hash(tmp_path, monkeypatch):
    at = tmp_path / "paper_2603_14371_amd" / "csrc"
    at.mkdir(parents=True)
    for name in bench.KERNEL_SOURCES:
        (at / name).write_bytes(open(os.path.join(CSRC, name), "rb").read())
    now = bench.kernel_source_hash()
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    assert bench.kernel_source_hash() == now
    for name in bench.KERNEL_SOURCES:
        old = (at / name).read_bytes()
        (at / name).write_bytes(old + b"\n")
        assert bench.kernel_source_hash() != now, name
        (at / name).write_bytes(old)


def test_the_figures_and_their_account_carry_one_stamp():
    with open(os.path.join(bench.ROOT, "profiles", "pmc_traffic_stress.json")) as f:
        stamp = json.load(f)["kernel_source_sha256_16"]
    with open(os.path.join(bench.ROOT, "profiles", "attn_kernel_stress_pmc_traffic.txt")) as f:
        assert stamp in f.read()
