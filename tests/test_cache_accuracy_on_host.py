"""The attention over the quantized cache on the host, thread by thread and under the sanitizers, on what a cache of real streams
holds: frames whose values, keys and queries are of very different sizes, in every form of the kernels, against float64 loops."""
import os
import subprocess

import pytest

from test_cache_on_host import spliced
from test_kernels_on_host import HERE, ROOT


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    path = tmp_path_factory.mktemp("cache_accuracy")
    src = spliced()
    rsq = "inline float __builtin_amdgcn_rsqf(float x) { return 1.0f / sqrtf(x); }"
    assert rsq in src          # the instruction takes operands below 2^-126 for zeros
    src = src.replace(rsq, rsq.replace("return", "if (x < 0x1p-126f) x = 0.0f; return"))
    src = "#include <string>\n" + src[:src.rindex("int main(")] + open(os.path.join(HERE, "host_emulation", "cache_accuracy_driver.cpp")).read()
    (path / "cache.cpp").write_text(src)
    r = subprocess.run(["g++", "-O0", "-g1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
                        "-std=c++20", "-pthread", "-I", os.path.join(HERE, "host_emulation"), "-I", os.path.join(ROOT, "include"),
                        str(path / "cache.cpp"), "-o", str(path / "cache")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return str(path / "cache")


@pytest.mark.parametrize("what", ["weights", "nonfinite", "scores", "queries", "gains", "sizes"])
def test_as_the_formula_says(exe, what):
    r = subprocess.run([exe, what], capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"), timeout=900)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.stdout[-3000:], r.stderr[-3000:])
