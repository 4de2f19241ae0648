"""The argument checks of a decoder layer's operators under AddressSanitizer and UBSan: the
CPU-only build of the host library runs test_ops_layer_abi.py in a subprocess with the
sanitizer runtimes preloaded."""
import os
import subprocess
import sys

import pytest

from paper_2607_11262_amd import build
from test_sanitizers import runtime

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.slow
def test_layer_argument_checks_under_asan_ubsan(tmp_path):
    host = build.build_host_sanitized(str(tmp_path / "libgts_host_san.so"))
    env = dict(os.environ)
    env.update(LD_PRELOAD=f"{runtime('libasan.so')}:{runtime('libubsan.so')}",
               ASAN_OPTIONS=f"detect_leaks=0:halt_on_error=1:log_path={tmp_path / 'asan'}",
               UBSAN_OPTIONS=f"halt_on_error=1:print_stacktrace=1:log_path={tmp_path / 'ubsan'}",
               GTS_TEST_SANITIZED_HOST=host)
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(HERE, "test_ops_layer_abi.py"), "-x", "-q", "-p",
                        "no:cacheprovider"], cwd=os.path.dirname(HERE), env=env, capture_output=True, text=True,
                       timeout=600)
    reports = "".join(open(tmp_path / f).read()[:4000] for f in sorted(os.listdir(tmp_path))
                      if f.startswith(("asan", "ubsan")))
    assert not reports, reports
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    mapped = [line for line in (r.stdout + r.stderr).splitlines() if line.startswith("[sanitized] mapped:")]
    assert mapped and host in mapped[0], (r.stdout + r.stderr)[-2000:]
