"""Build liballegro_latent.so (the operators of the latent track) in-tree.

The library stands beside liballegro_tp.so: it shares no kernel with it, needs no plan, and is built
with the same compiler flags.  Its two HIP sources are compiled at the same time, then linked; the
per-kernel register report goes to _build/latent_resource_usage.txt, and a kernel that spills to
scratch fails the build, as in build.py.
"""

from __future__ import annotations

import importlib.util
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(PKG, "liballegro_latent.so")
HIP_SOURCES = ("latent_rows.hip", "latent_matmul.hip")


def _base():
    """build.py, without importing the package (which needs the built libraries)."""
    spec = importlib.util.spec_from_file_location("_allegro_build", os.path.join(PKG, "build.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def build(verbose: bool = False) -> str:
    b = _base()
    os.makedirs(b.BUILD, exist_ok=True)
    objs = [os.path.join(b.BUILD, src.replace(".hip", ".o")) for src in HIP_SOURCES]
    jobs = [subprocess.Popen([b.HIPCC, *b.HIP_FLAGS, "-Rpass-analysis=kernel-resource-usage", "-c",
                              os.path.join(b.CSRC, src), "-o", obj], stdout=subprocess.PIPE,
                             stderr=subprocess.STDOUT, text=True) for src, obj in zip(HIP_SOURCES, objs)]
    reports = [job.communicate()[0] for job in jobs]
    for src, job, report in zip(HIP_SOURCES, jobs, reports):
        if job.returncode != 0:
            sys.stderr.write(report)
            raise RuntimeError(f"build step failed: hipcc {src}")
    summary, spills = b._check_resources("".join(reports))
    with open(os.path.join(b.BUILD, "latent_resource_usage.txt"), "w") as f:
        f.write(summary)
    if spills:
        raise RuntimeError("kernels use scratch memory (see _build/latent_resource_usage.txt): " + ", ".join(spills))
    tmp = LIB + ".tmp"
    b._run([b.HIPCC, "--offload-arch=" + b.ARCH, "-shared", "-fPIC", *objs, "-o", tmp])
    os.replace(tmp, LIB)
    if verbose:
        print(summary)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
