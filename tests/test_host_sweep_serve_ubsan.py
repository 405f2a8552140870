"""CPU-only: the host code of the quantized attention block's calls (argument checks, planners, workspace sizes, grid
arithmetic) compiled for the host alone under -fsanitize=undefined and driven over degenerate shapes by
tests/host_sweep_serve.cpp."""
import concurrent.futures as cf
import os
import shutil
import subprocess
import tempfile

import pytest

from test_host_sweep_ubsan import CSRC, FLAGS, HIPCC, ROOT, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_serving_host_code_under_ubsan():
    tmp = tempfile.mkdtemp(prefix="crvq_ubsan_")
    try:
        jobs = [[HIPCC] + FLAGS + ["-c", os.path.join(CSRC, f), "-o", f.replace(".hip", ".o")]
                for f in sorted(os.listdir(CSRC)) if f.endswith(".hip")]
        jobs.append([HIPCC] + FLAGS + ["-x", "hip", "-c", os.path.join(ROOT, "tests", "host_sweep_serve.cpp"), "-o", "sweep.o"])
        with cf.ThreadPoolExecutor(max_workers=4) as ex:
            list(ex.map(lambda c: _run(c, tmp), jobs))
        objs = sorted(f for f in os.listdir(tmp) if f.endswith(".o"))
        syms = sorted({ln.split()[-1] for ln in _run(["nm", "-u"] + objs, tmp).splitlines() if "__hip_fatbin_" in ln})
        with open(os.path.join(tmp, "fatbin_stub.c"), "w") as f:
            for s in syms:
                f.write(f"char {s}[4096] __attribute__((aligned(4096))) = {{0}};\n")
        _run(["gcc", "-c", "fatbin_stub.c", "-o", "fatbin_stub.o"], tmp)
        _run([HIPCC, "-Xarch_host", "-fsanitize=undefined", "-o", "sweep"] + objs +
             ["fatbin_stub.o", "-L/opt/rocm/lib", "-lrocprofiler-sdk-roctx", "-Wl,-rpath,/opt/rocm/lib"], tmp)
        r = subprocess.run(["./sweep"], cwd=tmp, capture_output=True, text=True, timeout=300,
                           env=dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1"))
        assert r.returncode == 0 and "host sweep ok" in r.stdout and "runtime error" not in r.stderr, r.stdout + r.stderr
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
