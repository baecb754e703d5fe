"""The host code of the model side of a step (argument checks, scratch sizes, launch set-up) built with AddressSanitizer and
UndefinedBehaviorSanitizer and walked by a small C driver (tests/host_checks/model_side_driver.c).  Nothing is launched, so no GPU is
needed."""
import importlib.util
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_host_code_of_the_model_side_under_asan_and_ubsan(tmp_path):
    spec = importlib.util.spec_from_file_location("_sv_build", os.path.join(ROOT, "paper_2509_24328_amd", "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    lib, exe = str(tmp_path / "libsv_san.so"), str(tmp_path / "model_side_driver")
    flags = [f for f in mod.FLAGS if f not in ("-O3", "-shared")] + ["-O1"]
    sources = [f"{n}.hip" for n in ("attention", "attention_bf16", "attention_bf16_f8", "attention_f32", "attention_f32_f8", "rope", "kv_cache",
                                    "sample", "api")]

    def compiled(name):
        out = str(tmp_path / (name + ".o"))
        return out, subprocess.run([HIPCC] + flags + san + ["-c", os.path.join(mod.CSRC, name), "-o", out], capture_output=True, text=True)

    with ThreadPoolExecutor(4) as pool:
        objects = list(pool.map(compiled, sources))
    for _, r in objects:
        assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared"] + san + ["-o", lib] + [o for o, _ in objects], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([HIPCC, "-x", "c", os.path.join(ROOT, "tests", "host_checks", "model_side_driver.c"), "-x", "none",
                        "-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-g",
                        "-o", exe, lib, f"-Wl,-rpath,{tmp_path}"], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out
    assert "host walk ok" in out and "runtime error" not in out and "AddressSanitizer" not in out, out
