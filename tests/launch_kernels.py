"""Builds and runs tests/launch_kernels_driver.cpp: which kernels a call of the operators around the linear layer launches."""
import os
import subprocess

from paper_2407_08296_amd import build as qg_build
from paper_2407_08296_amd import qgalore as qg

HERE = os.path.dirname(os.path.abspath(__file__))


def make(folder):
    """Returns run(calls): per call, a list of (kernel, workgroups in x, in y, threads); calls are tuples of a name and numbers."""
    qg.lib()
    exe = os.path.join(str(folder), "launch_kernels_driver")
    lib_dir = os.path.dirname(os.path.abspath(qg.LIB_PATH))
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "c++", "-std=c++17", "-O1",
                    "-I", os.path.join(qg_build.ROOT, "include"), os.path.join(HERE, "launch_kernels_driver.cpp"), "-rdynamic",
                    "-L", lib_dir, "-l:" + os.path.basename(qg.LIB_PATH), "-Wl,-rpath," + lib_dir, "-o", exe], check=True)

    def run(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        p = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300)
        assert p.returncode == 0, p.stdout[-500:] + p.stderr
        out, now = [], []
        for line in p.stdout.splitlines():
            if line.startswith("="):
                assert line == "= 0", (calls[len(out)], line)
                out.append(now)
                now = []
            else:
                name, sizes = line.split(" | ")
                now.append((name.replace("void ", "").replace("qg::", ""), *map(int, sizes.split())))
        assert len(out) == len(calls)
        return out
    return run
