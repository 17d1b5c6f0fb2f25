"""The microscaled calls' host code (checks, plans, workspace sizes) under
AddressSanitizer and UndefinedBehaviorSanitizer, as tests/test_sanitize.py does for the
other headers: their CPU tests run against the instrumented library in a child process."""

import os
import subprocess
import sys

from tests._util import ROOT


def _sanitized(build):
    """The instrumented library; built where it is missing or older than a source."""
    dirs = (build.CSRC, os.path.join(ROOT, "include"))
    newest = max(os.path.getmtime(f) for f in [build.__file__, *(os.path.join(d, n) for d in dirs for n in os.listdir(d))])
    if os.path.exists(build.SAN_LIB) and os.path.getmtime(build.SAN_LIB) > newest:
        return build.SAN_LIB
    return build.build_sanitized()


def test_microscaled_validation_under_asan_and_ubsan():
    from paper_2607_14107_amd import build
    lib = _sanitized(build)
    rt = build.asan_runtime()
    env = dict(os.environ)
    env.update(POLESTAR_LIB=lib, LD_PRELOAD=rt,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_mx_pins.py"), os.path.join(ROOT, "tests", "test_mx_plans.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    report = r.stdout[-3000:] + r.stderr[-3000:]
    assert r.returncode == 0, report
    assert "runtime error" not in report and "AddressSanitizer" not in report, report
    assert " passed" in r.stdout, report
