"""What the calls over a 4-bit cache would launch, recorded on the CPU as launch_record does it for the bfloat16 calls: the
host side of both is compiled with launchers that write down their arguments."""
import ctypes
import functools
import hashlib
import os
import subprocess
import tempfile

import launch_record as R
from paper_2402_14808_amd import build

SOURCES = ["relay_attn.hip", "cache_calls.hip"]


def _with(text, *edits):
    for old, new in edits:
        assert text.count(old) == 1, old
        text = text.replace(old, new)
    return text


LAUNCHERS = _with(
    R.LAUNCHERS,
    ('{"rows_sys", a.n_sys_rowblocks > 0},', '{"rows_sys", a.n_sys_rowblocks > 0}, {"fp4", a.fp4}, {"exact", a.exact}, '
     '{"prompts", a.cu_seqlens_q != nullptr}, {"batch", a.batch}, {"sys_wg_tiles", a.sys_wg_tiles}, '
     '{"sys_tiles", a.sys_tiles_total}, {"max_ctx", a.max_ctx}, {"cap", a.ctx_t_cap},'),
    ('{"part", a.ctx_part},', '{"part", a.ctx_part}, {"fp4", a.fp4}, {"exact", a.exact},'),
    ('hipError_t launch_relay_tiles', '''hipError_t launch_decode_direct_fp4(const DirectArgs &a, const DirectOne &, int, hipStream_t) {
    return add("direct_fp4", {{"tokens", a.n_tokens}}), hipSuccess;
}
hipError_t launch_fp4_rows(const Fp4RowsArgs &a, int, bool read, hipStream_t) {
    return add("fp4_rows", {{"tokens", a.n_tokens}, {"read", read}, {"slots", a.n_slots}}), hipSuccess;
}
hipError_t launch_update_tables(const TableArgs &a, hipStream_t) { return add("tables", {{"slots", a.n_slots}}), hipSuccess; }
hipError_t launch_relay_tiles'''))


@functools.lru_cache(1)
def library():
    text = LAUNCHERS + "".join(open(os.path.join(build.CSRC, f)).read() for f in SOURCES + build.HEADERS)
    name = hashlib.sha256((text + " ".join(build.FLAGS)).encode()).hexdigest()[:16]
    out = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_build", "fp4_launches_%s.so" % name)
    if not os.path.exists(out):
        os.makedirs(os.path.dirname(out), exist_ok=True)
        with tempfile.TemporaryDirectory(dir=os.path.dirname(out)) as tmp:
            src, new = os.path.join(tmp, "launchers.hip"), os.path.join(tmp, "recorded.so")
            with open(src, "w") as f:
                f.write(LAUNCHERS)
            r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")] + build.FLAGS + ["-Wl,-Bsymbolic", "-I", build.CSRC] +
                               [os.path.join(build.CSRC, f) for f in SOURCES] + [src, "-o", new], capture_output=True, text=True)
            assert r.returncode == 0, r.stderr[-2000:]
            for old in os.listdir(os.path.dirname(out)):
                if old.startswith("fp4_launches_"):
                    os.unlink(os.path.join(os.path.dirname(out), old))
            os.replace(new, out)
    lib = ctypes.CDLL(out)
    lib.take_launches.restype = ctypes.c_char_p
    for f in (lib.relay_attn_workspace_bytes, lib.relay_attn_workspace_bytes_fp4):
        f.restype = ctypes.c_size_t
    return lib


def workspace_bytes(p, total_q=None, fp4=True):
    lib = library()
    f = lib.relay_attn_workspace_bytes_fp4 if fp4 else lib.relay_attn_workspace_bytes
    return int(f(ctypes.byref(p), p.batch if total_q is None else total_q))


def decode(p, workspace=None):
    lib = library()
    size = R.SIZE(workspace_bytes(p) if workspace is None else workspace)
    return R._launches(lib, lib.relay_attn_decode_fp4(ctypes.byref(p), *[R.AT] * 10, size, None))


def prefill(p, total_q, max_q, workspace=None):
    lib = library()
    size = R.SIZE(workspace_bytes(p, total_q) if workspace is None else workspace)
    return R._launches(lib, lib.relay_attn_prefill_fp4(ctypes.byref(p), R.AT, R.AT, total_q, max_q, *[R.AT] * 9, size, None))
