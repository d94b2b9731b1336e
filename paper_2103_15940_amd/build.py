"""Builds libfmt.so (the C-ABI library, hand-written HIP for gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfmt.so")
SOURCES = ["fmt_api.hip", "fmt_stream.hip", "fmt_gemm.hip", "fmt_product_0.hip", "fmt_product_1.hip", "fmt_product_2.hip",
           "fmt_product_3.hip", "fmt_product_window.hip", "fmt_direct.hip", "fmt_fmac8.hip", "fmt_linear.hip", "fmt_dls.hip",
           "fmt_dropout.hip", "fmt_norm_fwd.hip", "fmt_norm_bwd.hip", "fmt_attention_fwd.hip", "fmt_attention_fwd_64.hip", "fmt_attention_fwd_128.hip", "fmt_attention_few.hip", "fmt_attention_bwd.hip",
           "fmt_attention_bwd_64.hip", "fmt_attention_bwd_128.hip"]
# packed-fp32 instructions (v_pk_add_f32 and friends) are kept out of the generated code on purpose:
# the rounding relies on every fp32 addition being one correctly rounded scalar operation
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wextra", "-Wno-unused-parameter",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = False, extra_flags=(), output: str = LIB, tag: str = "") -> str:
    """Compile every HIP source for gfx950 and link libfmt.so next to this file (or to `output`,
    with object files suffixed by `tag`, for tuning builds with extra -D flags)."""
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".hip", tag + ".o"))
        cmd = [hipcc(), *FLAGS, *extra_flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
               "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines()
                        if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
        if p.returncode != 0:
            failed = True
            sys.stderr.write("hipcc failed on %s:\n%s\n" % (src, out))
        elif verbose and out.strip():
            print(out)
    if failed:
        raise RuntimeError("libfmt build failed")
    tmp = output + ".tmp.%d" % os.getpid()
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, output)
    return output


if __name__ == "__main__":
    print(build(verbose=True))
