"""Builds libhfxattn.so for gfx950 with hipcc, in-tree next to this file."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhfxattn.so")
# The name says for which Python it was built, so that another one does not load it.
CALL_LIB = os.path.join(HERE, "_hfxcall" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = ["hfx_kernels.hip", "hfx_append.hip", "hfx_mx.hip", "hfx_api.cpp", "hfx_plan.cpp", "hfx_sched.cpp"]
# Sources with attention kernels, and their own flag.  -fno-honor-nans: without it every max of a softmax carries a canonicalising twin.  Nothing in them asks a
# floating-point operation whether a value is NaN: scores that may be (of unused slots, which hold anything) are masked, and weights that may be are told apart, by integer
# operations on bits that the compiler cannot see through.  Not for the appends over a projection's output, which may hold anything and of which that is asked.
# Device code only: the host side validates its floating-point arguments with NaN tests.
ATTENTION = ("hfx_kernels.hip", "hfx_mx.hip")
ATTENTION_FLAGS = ["-Xarch_device", "-fno-honor-nans"]
# The atomic optimizer is switched off: it rewrites thread 0's ticket fetch into a form that
# waits for the counter's reply on the spot, and the reply is only needed an item later.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _checked(ran) -> str:
    """What the compiler had to say, for (process, stderr) pairs; raises if one failed."""
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for _, text in ran for l in text.splitlines() if noise not in l)
    if any(p.returncode != 0 for p, _ in ran):
        raise RuntimeError("hipcc failed:\n" + err)
    return err


def build(verbose: bool = False, extra_flags=()) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects, commands = [], []
        for s in SOURCES:
            objects.append(os.path.join(tmp, s + ".o"))
            commands.append([hipcc, *FLAGS, *(ATTENTION_FLAGS if s in ATTENTION else ()), *extra_flags, "-c", "-o", objects[-1],
                             *(["-x", "hip"] if s.endswith(".cpp") else []), os.path.join(CSRC, s)])
        link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objects]
        if verbose:
            print("\n".join(" ".join(c) for c in commands + [link]), flush=True)
        running = [subprocess.Popen(c, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True) for c in commands]
        err = _checked([(p, p.communicate()[1]) for p in running])
        res = subprocess.run(link, capture_output=True, text=True)
        err += _checked([(res, res.stderr)])
    if verbose and err.strip():
        print(err, file=sys.stderr)
    build_call(verbose)
    return LIB


def build_call(verbose: bool = False) -> str:
    """The extension that marshals the arguments of the calls a serving loop makes (csrc/hfx_call.c)."""
    cmd = [os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-o", CALL_LIB,
           os.path.join(CSRC, "hfx_call.c")]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    untagged = os.path.join(HERE, "_hfxcall.so")      # of an earlier build, which any Python would load
    if os.path.exists(untagged):
        os.remove(untagged)
    if res.returncode != 0:
        raise RuntimeError("the call extension did not build:\n" + res.stderr)
    return CALL_LIB


if __name__ == "__main__":
    print(build(verbose=True))
