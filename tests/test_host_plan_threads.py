"""daris_free_plan on another thread than the other calls, under AddressSanitizer.  No GPU."""
import os
import subprocess

from test_host_sanitizers import CSRC, HERE, SAN, driver  # noqa: F401 (a fixture, which builds the library's sources)


def test_plans_may_be_freed_while_the_library_shuts_down(driver, tmp_path):  # noqa: F811
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    main, exe = os.path.join(HERE, "host_steps", "threads.cpp"), str(tmp_path / "threads")
    objs = []
    for name in ("aql.cpp", "launch.cpp", "sched_core.cpp", "net_plan.cpp", "net_encode.cpp", "daris_api.cpp"):
        o = os.path.join(HERE, "host_sanitize", name + ".san.o")
        if not os.path.exists(o) or os.path.getmtime(o) < os.path.getmtime(os.path.join(CSRC, name)):
            subprocess.check_call([hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-omit-frame-pointer"] + SAN + ["-c", os.path.join(CSRC, name), "-o", o],
                                  stderr=subprocess.DEVNULL)
        objs.append(o)
    subprocess.check_call([hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950"] + SAN + ["-c", main, "-o", exe + ".o"], stderr=subprocess.DEVNULL)
    subprocess.check_call([hipcc, "--offload-arch=gfx950"] + SAN + ["-o", exe, exe + ".o"] + objs +
                          [os.path.join(CSRC, "kernels_blob.o"), os.path.join(CSRC, "static_scratch.hip.o"), "-L/opt/rocm/lib", "-lhsa-runtime64", "-lpthread", "-ldl"], stderr=subprocess.DEVNULL)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:exitcode=23", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1:exitcode=24")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, f"exited with {r.returncode}:\n{r.stderr[-3000:]}"
    refused, unknown, other = map(int, r.stdout.split())
    assert refused + unknown > 0 and other == 0
