"""As test_host_sanitizers, for the entry points of the paged cache, of the attention over it and of the log-probabilities: tests/sanitize_generation_driver.c, linked with the
library's sources built with AddressSanitizer and UndefinedBehaviorSanitizer on the host side, has to run clean.  No GPU is touched."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]


def test_argument_validation_runs_clean_under_asan_and_ubsan(tmp_path):
    from paper_2602_08387_amd import build as b
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = [f for f in b.FLAGS if f != "-O3"] + ["-O1", "-g"]
    procs, objs = [], []
    for src in b.SOURCES:
        objs.append(str(tmp_path / src.replace(".hip", ".o")))
        procs.append(subprocess.Popen([hipcc, *flags, *san, "-c", os.path.join(b.CSRC, src), "-o", objs[-1]],
                                      stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for p in procs:
        out, _ = p.communicate()
        assert p.returncode == 0, out[-3000:]
    host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    driver, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    _run([hipcc, "-x", "c", "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-fno-gpu-sanitize", "-c",
          os.path.join(ROOT, "tests", "sanitize_generation_driver.c"), "-o", driver])
    _run([hipcc, "--offload-arch=gfx950", *host, "-fno-gpu-sanitize", *objs, driver, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    assert "all calls rejected as expected" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]
