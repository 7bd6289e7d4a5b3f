"""The planner's work lists under windows and prefix masks (tests/native/shaped_plans.cpp, compiled here
against the library; runs without a GPU)."""
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
PKG = os.path.join(ROOT, "paper_2606_16824_amd")


def test_plans_with_key_limits(tmp_path):
    exe = str(tmp_path / "shaped_plans")
    # (-fpermissive: the planner's headers name device builtins in templates that only kernels use)
    cmd = [shutil.which("g++") or "g++", "-std=c++17", "-O1", "-fpermissive", "-w", "-D__HIP_PLATFORM_AMD__", "-I",
           os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), "-I", "/opt/rocm/include",
           os.path.join(HERE, "native", "shaped_plans.cpp"), "-L", PKG, "-lcw", "-L", "/opt/rocm/lib", "-lamdhip64",
           f"-Wl,-rpath,{PKG}", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    print(r.stdout)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stderr
