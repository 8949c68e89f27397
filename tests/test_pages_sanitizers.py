"""The host side of the calls on 8-bit pages under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): lists of copies with a fault
anywhere, sizes and strides at the ends of their types."""
import glob
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_host_sanitizers import COMMON, HIPCC, HOST_SAN, ROOT, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc in this environment")
def test_calls_on_pages_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    sources = sorted(glob.glob(os.path.join(ROOT, "paper_2603_05353_amd", "csrc", "*.hip")))
    sources.append(os.path.join(ROOT, "tests", "host_pages_sanitized.cpp"))
    objects = [str(tmp_path / (os.path.splitext(os.path.basename(s))[0] + ".o")) for s in sources]
    with ThreadPoolExecutor(max_workers=8) as pool:
        for src, r in zip(sources, pool.map(lambda p: _run([HIPCC] + COMMON + HOST_SAN + ["-c", p[0], "-o", p[1]]), zip(sources, objects))):
            assert r.returncode == 0, f"{src}:\n{r.stderr[-3000:]}"
    exe = str(tmp_path / "host_pages_sanitized")
    r = _run([HIPCC, "-fsanitize=address", "-fsanitize=undefined"] + objects + ["-o", exe])
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = _run([exe], env=env, timeout=300)
    assert r.returncode == 0, f"stdout:\n{r.stdout[-3000:]}\nstderr:\n{r.stderr[-3000:]}"
    assert "calls on pages under the sanitizers: ok" in r.stdout
    assert "Sanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-3000:]
