"""The host code of the few-bit calls under AddressSanitizer and UndefinedBehaviorSanitizer (CPU).

Builds the library's host code and the stand-in of the HIP runtime with both, and runs the tests of
the few-bit calls' host code on that build in a child process with the sanitizers' runtime
preloaded.  Any report fails the test."""
import glob
import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest

import standin

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OUT = os.path.join(ROOT, "_build", "standin_sanitize")

pytestmark = pytest.mark.spawns

MODULES = ["tests/test_mx_host.py", "tests/test_mx_tables.py", "tests/test_mx_tiles_host.py",
           "tests/test_mx_overlap.py", "tests/test_mx_plan.py"]

CHILD = """
import sys
sys.path[:0] = [{tests!r}, {root!r}]
import standin
standin.build = lambda: {lib!r}
import pytest
sys.exit(pytest.main([*{modules!r}, "-q", "-x", "-p", "no:cacheprovider", "-k", "not plain_c"]))
"""


def build(b):
    os.makedirs(OUT, exist_ok=True)
    sources = [os.path.join(standin.HERE, "hip_standin.cpp")] + [os.path.join(standin.CSRC, s) for s in b.SOURCES]
    objs = [os.path.join(OUT, os.path.basename(s) + ".o") for s in sources]
    flags = ["-O1" if f == "-O3" else f for f in b.COMMON] + b.SANITIZE_HOST
    jobs = [[b.HIPCC, f"--offload-arch={b.ARCH}", *flags, "-x", "hip", "--cuda-host-only", "-c", s, "-o", o]
            for s, o in zip(sources, objs)]
    with ThreadPoolExecutor(max_workers=8) as ex:
        list(ex.map(b._run, jobs))
    undefined = subprocess.run(["nm", "-u", *objs], stdout=subprocess.PIPE, text=True, check=True).stdout
    lib = os.path.join(OUT, "libcosta_standin.so")
    # (the sanitizers' own symbols come with the preloaded runtime)
    b._run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", lib, *objs,
            *[f"-Wl,--defsym,{s}=0" for s in sorted(set(re.findall(r"__hip_fatbin\w*", undefined)))], "-lpthread"])
    return lib


@pytest.mark.slow
def test_few_bit_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    b = standin._by_path("costa_build", os.path.join(ROOT, "paper_2106_06601_amd", "build.py"))
    lib = build(b)
    log = str(tmp_path / "san")
    opts = f"halt_on_error=1:log_path={log}"
    env = dict(os.environ, LD_PRELOAD=b.sanitizer_runtime(), COSTA_LIB=lib,
               ASAN_OPTIONS="detect_leaks=0:" + opts, UBSAN_OPTIONS="print_stacktrace=1:" + opts)
    child = CHILD.format(tests=os.path.join(ROOT, "tests"), root=ROOT, lib=lib, modules=MODULES)
    r = subprocess.run([sys.executable, "-c", child], cwd=ROOT, env=env, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=900)
    reports = sorted(glob.glob(log + "*"))
    text = "".join(open(f).read()[:4000] for f in reports)
    assert not reports, f"sanitizer reports:\n{text}"
    assert r.returncode == 0, r.stdout[-4000:]
