"""Builds the HIP library for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
LIB_PATH = os.path.join(_HERE, "libqsl.so")
# two translation units in folders of their own: the compression path, and the operators on a model's logits
SOURCES = [os.path.join(_HERE, "csrc", "qsl.hip"), os.path.join(_HERE, "csrc_logits", "logits.hip")]
HEADERS = [os.path.join(_HERE, "csrc", h) for h in ("qsl_policy.h", "qsl_device.h", "qsl_layout.h", "qsl_stream.h", "qsl_select.h",
                                                    "qsl_encode.h", "qsl_lean.h", "qsl_whole.h", "qsl_window.h", "qsl_dense.h",
                                                    "qsl_decode.h")] + [os.path.join(_HERE, "csrc_logits", "qsl_logits.h"),
                                                        os.path.join(ROOT, "include", "qsl.h")]

HIPCC_FLAGS = [
    "-O3", "--offload-arch=gfx950", "-std=c++17",
    "-ffp-contract=off",                                        # one rounding per written fp operation
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fPIC",
    "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(_HERE, "csrc"),
]


def build(verbose: bool = False) -> str:
    """Compile libqsl.so (always recompiles), the translation units side by side."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        jobs = [subprocess.Popen([hipcc] + HIPCC_FLAGS + ["-c", "-o", o, s], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                for s, o in zip(SOURCES, objects)]
        said = [job.communicate()[0] for job in jobs]
        if all(job.returncode == 0 for job in jobs):
            link = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB_PATH] + objects, capture_output=True, text=True)
            said.append(link.stdout + link.stderr)
            failed = link.returncode != 0
        else:
            failed = True
    if failed:
        raise RuntimeError("hipcc failed:\n" + "\n".join(said))
    if verbose:
        print("\n".join(said))
    return LIB_PATH


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS)


if __name__ == "__main__":
    print(build(verbose=True))
