"""Builds librelayattn.so (gfx950 HIP kernels + C ABI) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librelayattn.so")
SOURCES = ["relay_attn.hip", "relay_tiles.hip", "decode_direct.hip", "relay_rows.hip", "ctx_paged.hip", "fuse.hip", "validate.hip",
           "fp4_cache.hip", "fp4_direct.hip", "tables.hip", "cache_calls.hip"]
HEADERS = ["ra_device.h", "ra_kernels.h", "rows_item.h", "token_place.h", "fp4.h", "fp4_attend.h", "ra_host.h", "direct_kernel.h",
           os.path.join("..", "..", "include", "relay_attn.h")]

# -packed-fp32-ops off: scalar float code must not be fused into v_pk_*_f32 forms.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall",
         "-Wno-unused-command-line-argument", "-Wno-inline-asm"]


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [hipcc] + FLAGS + [os.path.join(CSRC, f) for f in SOURCES] + ["-o", tmp]
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err)
    # a library with an unresolved symbol builds fine but cannot be loaded: check now
    import ctypes
    try:
        ctypes.CDLL(tmp)
    except OSError as e:
        os.unlink(tmp)
        raise RuntimeError("built library does not load: %s" % e)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
