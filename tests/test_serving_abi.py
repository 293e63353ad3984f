"""Host code of the serving entry points (argument checks, workspace queries) under AddressSanitizer and UndefinedBehaviorSanitizer, on the
CPU, as tests/test_host_sanitizer.py does for the others; and the binding's structures against the header's."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2403_02352_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def build_script():
    import importlib.util
    spec = importlib.util.spec_from_file_location("_atp_build", os.path.join(ROOT, "paper_2403_02352_amd", "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_host_paths_under_address_and_ub_sanitizers(tmp_path):
    mod = build_script()
    objs = [os.path.join(CSRC, s.replace(".hip", ".o")) for s in mod.SOURCES if s != "api_serving.hip"]
    if not all(os.path.exists(o) for o in objs):
        mod.build_library(verbose=False)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
           "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wno-unused-command-line-argument"]
    api_o, drv_o, exe = (str(tmp_path / n) for n in ("api_san.o", "driver.o", "host_checks"))
    for cmd in ([HIPCC, *flags, *san, "-c", os.path.join(CSRC, "api_serving.hip"), "-o", api_o],
                [HIPCC, "-O1", "-g", "-std=c++17", "-x", "c++", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-c", os.path.join(ROOT, "tests", "serving_sanitizer_driver.cpp"), "-o", drv_o],
                [HIPCC, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", "-o", exe, drv_o, api_o, *objs]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    assert "host checks ok" in r.stdout


def test_structures_of_the_binding_match_the_header(tmp_path):
    from paper_2403_02352_amd import binding
    fields = {"atp_cache": binding._Cache, "atp_batch": binding._Batch}
    src = tmp_path / "layout.c"
    lines = [f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));' for n, s in fields.items() for f, _ in s._fields_]
    lines += [f'printf("{n} %zu\\n", sizeof({n}));' for n in fields]
    src.write_text(f'#include "{ROOT}/include/atp.h"\n#include <stdio.h>\nint main(void) {{ {" ".join(lines)} return 0; }}\n')
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "layout")], check=True)
    said = dict(line.split() for line in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines())
    for n, s in fields.items():
        assert int(said[n]) == C.sizeof(s)
        for f, _ in s._fields_:
            assert int(said[f"{n}.{f}"]) == getattr(s, f).offset, f
