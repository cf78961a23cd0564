"""The launches of the calls around products with the host code under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU)."""
import glob
import os
import subprocess
import sys

import pytest

import standin
import test_mx_sanitizers as few_bit

pytestmark = pytest.mark.spawns


@pytest.mark.slow
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    b = standin._by_path("costa_build", os.path.join(few_bit.ROOT, "paper_2106_06601_amd", "build.py"))
    lib = few_bit.build(b)
    log = str(tmp_path / "san")
    opts = f"halt_on_error=1:log_path={log}"
    env = dict(os.environ, LD_PRELOAD=b.sanitizer_runtime(), COSTA_LIB=lib,
               ASAN_OPTIONS="detect_leaks=0:" + opts, UBSAN_OPTIONS="print_stacktrace=1:" + opts)
    child = few_bit.CHILD.format(tests=os.path.join(few_bit.ROOT, "tests"), root=few_bit.ROOT, lib=lib,
                                 modules=["tests/test_layer_calls.py"])
    child = child.replace("not plain_c", "not long_operands")  # (thousands of slices a call, each as the others)
    r = subprocess.run([sys.executable, "-c", child], cwd=few_bit.ROOT, env=env, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=900)
    text = "".join(open(f).read()[:4000] for f in sorted(glob.glob(log + "*")))
    assert not text, f"sanitizer reports:\n{text}"
    assert r.returncode == 0, r.stdout[-4000:]
