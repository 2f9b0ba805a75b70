"""Which kernels the calls of the 4-bit path and the routers by scores launch, found without a GPU (launches_host.cpp)."""
import os
import subprocess
from typing import NamedTuple

from paper_2605_17889_amd import build as hip_build

HERE = os.path.dirname(os.path.abspath(__file__))


class Launch(NamedTuple):
    kernel: str
    grid: int
    threads: int


def compile_program(folder) -> str:
    if not os.path.exists(hip_build.LIB):
        hip_build.build()
    out = os.path.join(str(folder), "launches_host")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(hip_build.ROOT, "include"), "-I", "/opt/rocm/include",
                    os.path.join(HERE, "launches_host.cpp"), "-o", out, hip_build.LIB,
                    "-Wl,-rpath," + os.path.dirname(hip_build.LIB), "-Wl,-rpath-link,/opt/rocm/lib"], check=True)
    return out


def run(program: str, calls):
    """[(status, [Launch, ..])] of the calls, one line each, in one process."""
    lines = iter(subprocess.run([program], input="".join(c + "\n" for c in calls), capture_output=True, text=True, timeout=120,
                                check=True).stdout.splitlines())
    out = []
    for _ in calls:
        status, n = map(int, next(lines).split())
        launches = (next(lines).rsplit("|", 2) for _ in range(n))
        out.append((status, [Launch(kernel, int(grid), int(threads)) for kernel, grid, threads in launches]))
    return out


def kernels(program: str):
    return subprocess.run([program], input="kernels\n", capture_output=True, text=True, timeout=120, check=True).stdout.splitlines()
