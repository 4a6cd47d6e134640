"""Builds libmassive.so (hipcc, gfx950) in-tree."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", name) for name in ("massive.hip", "operators.hip", "layers.hip")]
LIB = os.path.join(HERE, "libmassive.so")
ARCH = os.environ.get("MASSIVE_OFFLOAD_ARCH", "gfx950")

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=" + ARCH,
    # no packed-fp32 instructions anywhere in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # float atomicAdd as the native global atomic
    "-munsafe-fp-atomics",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp%d" % os.getpid()
    # the sources compile side by side
    objects = ["%s.%s.o" % (tmp, os.path.basename(src)) for src in SRCS]
    compiles = [["hipcc"] + [f for f in FLAGS if f != "-shared"] + ["-c", src, "-o", o] for src, o in zip(SRCS, objects)]
    link = ["hipcc", "-shared", "-fPIC", "--offload-arch=" + ARCH] + objects + ["-o", tmp]
    try:
        running = []
        for cmd in compiles:
            if verbose:
                print(" ".join(cmd), flush=True)
            running.append(subprocess.Popen(cmd))
        for cmd, status in zip(compiles, [p.wait() for p in running]):
            if status:
                raise subprocess.CalledProcessError(status, cmd)
        if verbose:
            print(" ".join(link), flush=True)
        subprocess.check_call(link)
        os.replace(tmp, LIB)
    finally:
        for f in objects + [tmp]:
            if os.path.exists(f):
                os.remove(f)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
