"""CPU build with AddressSanitizer and UndefinedBehaviorSanitizer of the host code
of dropout, the norm, the cross-entropy over many classes and the model with
dropout (hipcc, host side only), its launches ending in stand-ins: the plans'
arithmetic over the extents that the entry points take, and every launch's."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NATIVE = os.path.join(ROOT, "tests", "native")
CSRC = os.path.join(ROOT, "paper_2010_05337_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
         "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _run(cmd, **kw):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, **kw)
    assert r.returncode == 0, f"{' '.join(cmd[:3])} ... failed ({r.returncode}):\n{r.stdout[-4000:]}"
    return r.stdout


@pytest.mark.slow
@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc is not installed")
def test_head_host_code_under_sanitizers(tmp_path):
    sources = [os.path.join(CSRC, s) for s in ("linear_loss.hip", "rows.hip", "api_head.hip", "api.hip")]
    sources += [os.path.join(NATIVE, s) for s in ("abi_stubs.cpp", "head_sanitize_main.cpp")]
    objs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in sources]
    with ThreadPoolExecutor(max_workers=4) as ex:
        list(ex.map(lambda so: _run([HIPCC, *FLAGS, "-c", so[0], "-o", so[1]], cwd=str(tmp_path)), zip(sources, objs)))
    exe = str(tmp_path / "head_san")
    _run([HIPCC, *FLAGS, *objs, "-o", exe], cwd=str(tmp_path))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    assert "ok" in _run([exe], env=env, cwd=str(tmp_path))
