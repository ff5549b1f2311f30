"""The host half of include/sphattn_layer.h and of the distillation under AddressSanitizer and UndefinedBehaviorSanitizer: tests/sanitizers/layer_driver.cpp, no GPU
involved."""
import os
import subprocess

from test_sanitizers import ENV, SAN


def test_layer_host_code_under_asan_ubsan(tmp_path):
    from paper_2505_09326_amd._build import CSRC, HIPCC_FLAGS
    exe = str(tmp_path / "layer_driver")
    flags = [f for f in HIPCC_FLAGS if f not in ("-O3", "-shared", "-fPIC")]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-O1", "-g", "-Wno-inline-asm", *san, "-o", exe,
           os.path.join(CSRC, "sphattn_train.hip"), os.path.join(CSRC, "sphattn_layer.hip"), os.path.join(SAN, "layer_driver.cpp")]
    b = subprocess.run(cmd, capture_output=True, text=True)
    assert b.returncode == 0, b.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, env=ENV)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout + r.stderr)[-4000:]
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
