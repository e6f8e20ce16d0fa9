"""The host side of the layer operators under AddressSanitizer and UndefinedBehaviorSanitizer (gcc): a program walks through what
random calls are planned to do (tests/hip_stub/layer_plan.cpp), every access inside its tensor and every result written once."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "hip_stub")


def test_planned_accesses_of_random_calls(tmp_path):
    exe = str(tmp_path / "layer_plan")
    csrc = os.path.join(ROOT, "paper_2511_11062_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-Wall", "-Wextra", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-I" + STUB, "-I" + os.path.join(ROOT, "include"), "-I" + csrc, os.path.join(csrc, "lite_attn_layer_host.cpp"),
           os.path.join(STUB, "layer_plan.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert res.returncode == 0 and "layer plan ok" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]
