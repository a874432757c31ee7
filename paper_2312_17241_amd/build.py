"""Compile the HIP sources into paper_2312_17241_amd/libcngp.so for gfx950.

hipcc cross-compiles without a GPU.  Flags: packed fp32 instructions are switched off
(-packed-fp32-ops), floating-point atomics use the hardware instructions
(-munsafe-fp-atomics; all gradient buffers are ordinary coarse-grained device memory).
"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcngp.so")
SOURCES = ["cngp_api.hip", "cngp_sort.hip", "cngp_recur.hip", "cngp_recur_fwd.hip", "cngp_recur_bwd.hip", "cngp_embed.hip", "cngp_balance.hip"]
HEADERS = ["cngp_launch.h", "cngp_radix.h", "cngp_recur.h", "cngp_recur_scan.h", "cngp_device.h", "cngp_kernels.h", "cngp_fwd_level.h", "cngp_bwd_sliced.h", "cngp_bwd_binned.h", "cngp_bwd_merge.h", "cngp_bwd_runs.h", "cngp_optim.h", "cngp_mlp.h", "cngp_rates.h", os.path.join("..", "..", "include", "cngp.h")]

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-munsafe-fp-atomics",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function"]


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def _compile_and_link(flags, sources, out_dir, out, link_flags, what):
    """Every source to an object, side by side, then one link."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(out_dir, exist_ok=True)
    objects = [os.path.join(out_dir, os.path.basename(f) + ".o") for f in sources]
    jobs = [subprocess.Popen([hipcc] + flags + ["-c", "-o", o, f], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            for f, o in zip(sources, objects)]
    log = "".join(job.communicate()[0] for job in jobs)
    failed = any(job.returncode for job in jobs)
    if not failed:
        res = subprocess.run([hipcc] + link_flags + ["-o", out] + objects, capture_output=True, text=True)
        log, failed = log + res.stdout + res.stderr, res.returncode != 0
    msgs = [ln for ln in log.splitlines() if "packed-fp32-ops" not in ln]          # the host pass does not know the feature: harmless
    if failed:
        raise RuntimeError(f"{what} failed:\n" + "\n".join(msgs))
    return msgs


def build(force: bool = True, extra=()) -> str:
    if not force and not stale():
        return LIB
    out_dir = os.path.join(os.path.dirname(HERE), "_build")
    msgs = _compile_and_link([f for f in FLAGS if f != "-shared"] + list(extra), [os.path.join(CSRC, f) for f in SOURCES], out_dir, LIB,
                             ["--offload-arch=gfx950", "-shared", "-fPIC"], "hipcc")
    if msgs:
        print("\n".join(msgs), file=sys.stderr)
    return LIB


def build_host_sanitized() -> str:
    """The library's host code (validation, plan, workspace layout) with its exerciser csrc/host_check_main.cpp as one
    program, AddressSanitizer and UndefinedBehaviorSanitizer on the HOST side only (the device side is compiled as
    always; nothing of it runs).  About two minutes; the result lives in the git-ignored _build/ folder and is
    rebuilt only when a source is newer.  tests/test_abi.py runs it."""
    out_dir = os.path.join(os.path.dirname(HERE), "_build")
    os.makedirs(out_dir, exist_ok=True)
    exe = os.path.join(out_dir, "cngp_host_sanitize_check")
    main = os.path.join(CSRC, "host_check_main.cpp")
    srcs = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [main]
    if os.path.exists(exe) and os.path.getmtime(exe) >= max(os.path.getmtime(f) for f in srcs):
        return exe
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined"]
    flags = [f for f in FLAGS if f not in ("-shared", "-fPIC", "-O3")] + ["-O1", "-g"] + san
    _compile_and_link(flags, [main] + [os.path.join(CSRC, s) for s in SOURCES], os.path.join(out_dir, "sanitized"), exe,
                      ["--offload-arch=gfx950"] + san, "hipcc (host sanitizers)")
    return exe


def build_host_recur() -> str:
    """The recurrence's arithmetic that host and device share (csrc/cngp_recur.h) with its checks csrc/host_check_recur_main.cpp, for the host alone.
    The result lives in the git-ignored _build/ folder and is rebuilt when a source is newer.  tests/test_recur_host.py runs it."""
    out_dir = os.path.join(os.path.dirname(HERE), "_build")
    os.makedirs(out_dir, exist_ok=True)
    exe = os.path.join(out_dir, "cngp_host_check_recur")
    srcs = [os.path.join(CSRC, "host_check_recur_main.cpp")] + [os.path.join(CSRC, f) for f in ("cngp_recur.h", "cngp_launch.h")]
    if os.path.exists(exe) and os.path.getmtime(exe) >= max(os.path.getmtime(f) for f in srcs):
        return exe
    res = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "hip", "--offload-host-only", "-O2", "-std=c++17", "-Wall",
                          "-Wno-unused-function", "-o", exe, srcs[0]], capture_output=True, text=True)
    if res.returncode:
        raise RuntimeError("hipcc (host checks of the recurrence) failed:\n" + res.stdout + res.stderr)
    return exe


if __name__ == "__main__":
    if "--host-sanitizers" in sys.argv:
        print(build_host_sanitized())
    else:
        print(build(force=True, extra=sys.argv[1:]))
