"""Finding a kept plan allocates nothing on the host (tests/native/kept_plan_allocs.c, built by
build(); runs without a GPU)."""
import os
import subprocess

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native")


def test_kept_plans_are_found_without_allocating():
    exe = os.path.join(NATIVE, "kept_plan_allocs.bin")
    assert os.path.exists(exe), "tests/native/kept_plan_allocs.bin is missing: run __graft_entry__.build()"
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stderr
