"""Builds libdblp.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
import glob
import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libdblp.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + [os.path.join(ROOT, "include", "dblp.h")]


def registers(path=OUT):
    """Registers a thread of every kernel in a library built here, by mangled name; none where the toolkit has no tool for it (the launch
    looks as well)."""
    tool = os.path.join(os.path.dirname(NVCC), "cuobjdump")
    if not os.path.exists(tool):
        return {}
    text = subprocess.run([tool, "--dump-resource-usage", path], check=True, capture_output=True, text=True).stdout
    return {name: int(n) for name, n in re.findall(r"Function (\S+):\s+REG:(\d+)", text)}


def check_registers(found):
    """The products that sum in runs move registers between their warps, and refuse to start with another number than they count on."""
    with open(os.path.join(CSRC, "product_kernels.cuh")) as f:
        want = int(re.search(r"kRunRegs = (\d+)", f.read()).group(1))
    wrong = {name: n for name, n in found.items() if re.search(r"k_productILi\dELb1E", name) and n != want}
    if wrong:
        raise RuntimeError("kernels that would refuse to start, built with other than %d registers a thread: %s" % (want, wrong))


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(OUT) and all(os.path.getmtime(OUT) >= os.path.getmtime(f) for f in _deps()):
        return OUT
    cmd = [NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads", "0", "-shared",
           "-Xcompiler", "-fPIC,-Wall", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", OUT]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    made = OUT[:-3] + ".new.so"
    cmd[cmd.index(OUT)] = made
    subprocess.run(cmd + sources(), check=True)
    check_registers(registers(made))
    os.replace(made, OUT)
    return OUT


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
