"""Builds libactq.so in-tree with hipcc for gfx950 (cross-compiles without a GPU), and actq_torch.so, the
binding's native half, with the host compiler against torch's headers."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libactq.so")
SOURCES = ["actq_api.cpp", "actq_kernels.hip", "actq_context.hip", "actq_linear.hip", "actq_head_norm.hip", "actq_cache.hip", "actq_attention.hip", "actq_append.hip", "actq_block.hip",
           "actq_linear4.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # the scaling step of the quantizer is a separately rounded subtract and multiply
    "-ffp-contract=off",
    # inputs are finite by contract: lets min/max compile to single v_min/v_max (and fold
    # into DPP forms) instead of quieting signalling NaNs first
    "-fno-honor-nans",
    # keep binary32 arithmetic on the scalar-issue VALU forms
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
    # "#pragma unroll" on loops whose trip count is a template parameter that may be a run-time value
    "-Wno-pass-failed",
]


# sources with instructions of their own that read other lanes, for which the compiler does not wait
LANE_READERS = ["actq_attention.hip"]

HOST_LIB = os.path.join(_HERE, "actq_torch.so")
HOST_SOURCE = "actq_torch.cpp"
HOST_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
              "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM"]   # what torch's headers for this platform ask for


def _digest(files, *texts) -> str:
    import hashlib
    h = hashlib.sha256()
    for path in files:
        h.update(os.path.basename(path).encode())
        with open(path, "rb") as f:
            h.update(f.read())
    for text in texts:
        h.update(text.encode())
    return h.hexdigest()[:16]


def source_hash() -> str:
    """Digest of everything the library depends on: the sources, the public and internal headers
    and the compiler flags."""
    files = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith((".hip", ".cpp", ".h")) and f != HOST_SOURCE]
    return _digest(files + [os.path.join(ROOT, "include", "actq.h")], " ".join(HIPCC_FLAGS))


def host_source_hash() -> str:
    """The same for the binding's native half, which depends on the interpreter's binary interface and on torch's as well."""
    import sysconfig
    import torch
    return _digest([os.path.join(CSRC, HOST_SOURCE), os.path.join(CSRC, "actq_overlap.h"), os.path.join(ROOT, "include", "actq.h")], " ".join(HOST_FLAGS),
                   f"{sysconfig.get_config_var('SOABI')} torch {torch.__version__} {_abi_flag()}")


def _abi_flag() -> str:
    """The C++ library's interface that this torch was built with."""
    import torch
    return f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: libactq cannot be built")
    return exe


def _registers(operand: str) -> set:
    """The vector registers that an operand names: v7, v[4:7], |v7|, -v7."""
    m = re.fullmatch(r"[-|]*v(?:(\d+)|\[(\d+):(\d+)\])\|?", operand.strip())
    if not m:
        return set()
    return {int(m[1])} if m[1] else set(range(int(m[2]), int(m[3]) + 1))


def lane_read_hazards(assembly: str) -> list:
    """What is too near to the DPP multiply-adds in an assembly listing.  The compiler waits for the results of its own instructions; of those written by hand
    it knows the operands only.  A lane of another's register needs two wait states after a vector instruction has written it, the result of an exponential, a
    reciprocal and the like one before anything reads it, that of a matrix instruction up to 18 (unless one of the compiler's own has used it in between, which
    has waited for it), and lanes that a vector comparison has switched five.
    An instruction is a wait state, s_nop n is n + 1; what lies before a label is not known and counts as a hazard."""
    found, window = [], []   # of instructions since the last label: (wait states, mnemonic, registers written, registers used, whether it is one of ours)
    label = True
    for number, line in enumerate(assembly.splitlines(), 1):
        text = line.split(";")[0].split("//")[0].strip()
        if not text or text.startswith((".", "#")) and not text.endswith(":"):
            continue
        if text.endswith(":"):
            window, label = [], True
            continue
        name, _, rest = text.partition(" ")
        operands = re.split(r",\s*(?![^\[]*\])", rest.strip().split(" row_")[0]) if rest else []
        ours = name == "v_fmac_f32_dpp" and "row_newbcast" in text
        if ours:
            target, source, factor = (_registers(o) for o in operands[:3])
            waited, known = 0, set()
            for states, other, written, used, by_hand in reversed(window):
                trans = re.match(r"v_(exp|log|rcp|rsq|sqrt|sin|cos)_", other)
                matrix = other.startswith(("v_mfma", "v_smfmac"))
                if other.startswith("v_") and (waited < 2 and written & source or trans and waited < 1 and written & (source | factor | target)
                                               or matrix and waited < 18 and (written & (source | factor | target)) - known or other.startswith("v_cmpx") and waited < 5):
                    found.append(f"line {number}: {text}  behind {other}")
                waited += states
                known |= set() if by_hand else used
            if label and waited < 2:
                found.append(f"line {number}: {text}  behind a label")
        states = int(operands[0], 0) + 1 if name == "s_nop" else 1
        written = _registers(operands[0]) if name.startswith("v_") and operands else set()
        window = (window + [(states, name, written, set().union(*map(_registers, operands)) if name.startswith("v_") else set(), ours)])[-18:]
    return found


def build(verbose: bool = False) -> str:
    """Compile every source of the library; always recompiles."""
    from concurrent.futures import ThreadPoolExecutor
    tmp = LIB + f".{os.getpid()}.tmp"
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    noise = "'-packed-fp32-ops' is not a recognized feature"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)

    # one object per source, side by side: the largest takes as long as the others together
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as pool:
        common = [hipcc(), *flags, f'-DACTQ_SOURCE_HASH="{source_hash()}"', "-I", os.path.join(ROOT, "include"), "-I", CSRC]
        made = [os.path.join(objects, s + ".o") for s in SOURCES]
        listing = {s: ["-save-temps=obj"] if s in LANE_READERS else [] for s in SOURCES}
        for done in [pool.submit(run, [*common, *listing[s], "-x", "hip", "-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, made)]:
            done.result()
        for s in LANE_READERS:
            listings = [f for f in os.listdir(objects) if f.startswith(os.path.splitext(s)[0]) and "gfx950" in f and f.endswith(".s")]
            if len(listings) != 1:
                raise RuntimeError(f"{s}: no assembly listing to check")
            with open(os.path.join(objects, listings[0])) as f:
                hazards = lane_read_hazards(f.read())
            if hazards:
                raise RuntimeError(f"{s}: lanes read too early:\n" + "\n".join(hazards[:20]))
        run([hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", *made, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


def build_host(verbose: bool = False) -> str:
    """Compile the binding's native half; always recompiles."""
    import sysconfig
    import torch
    where = os.path.dirname(torch.__file__)
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("no C++ compiler: actq_torch cannot be built")
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(hipcc())))
    tmp = HOST_LIB + f".{os.getpid()}.tmp"
    cmd = [cxx, *HOST_FLAGS, f'-DACTQ_SOURCE_HASH="{host_source_hash()}"', _abi_flag()]
    for path in (os.path.join(ROOT, "include"), os.path.join(where, "include"), os.path.join(where, "include", "torch", "csrc", "api", "include"),
                 os.path.join(rocm, "include"), sysconfig.get_paths()["include"]):
        cmd += ["-isystem" if path.startswith(where) else "-I", path]
    cmd += [os.path.join(CSRC, HOST_SOURCE), "-o", tmp, "-L" + os.path.join(where, "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu", "-ltorch", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cxx} failed:\n{r.stderr}")
    if verbose and r.stderr.strip():
        print(r.stderr, file=sys.stderr)
    os.replace(tmp, HOST_LIB)
    return HOST_LIB


if __name__ == "__main__":
    print(build(verbose=True))
    print(build_host(verbose=True))
