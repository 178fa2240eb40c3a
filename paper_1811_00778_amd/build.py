"""Build libhcnn.so (HIP, gfx950) in-tree: `python -m paper_1811_00778_amd.build`."""
import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_DIR = os.path.join(_HERE, "lib")
LIB = os.path.join(LIB_DIR, "libhcnn.so")
SOURCES = [os.path.join(CSRC, s) for s in ("hcnn.cpp", "plain.cpp", "plain_f32.cpp", "plain_f16.cpp", "plain_bf16.cpp")]
HEADERS = [os.path.join(CSRC, h) for h in ("platform.h", "modarith.h", "ntt_kernels.h", "fv_kernels.h", "rate_kernels.h", "plain_kernels.h", "plain_host.h")]
HEADERS.append(os.path.join(os.path.dirname(_HERE), "include", "hcnn.h"))

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed FP32 instructions are kept out of every kernel of this library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-parameter",
]


def up_to_date() -> bool:
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(f) <= t for f in SOURCES + HEADERS)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(LIB_DIR, exist_ok=True)
    tmp = LIB + ".tmp.%d" % os.getpid()
    objects = [tmp + "." + os.path.basename(src) + ".o" for src in SOURCES]
    commands = [["hipcc"] + HIPCC_FLAGS + ["-x", "hip", "-c", src, "-o", obj] for src, obj in zip(SOURCES, objects)]
    link = ["hipcc", "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp] + objects
    if verbose:
        print("\n".join(" ".join(c) for c in commands + [link]))
    try:
        running = [subprocess.Popen(c) for c in commands]           # the translation units side by side
        codes = [p.wait() for p in running]
        for c, code in zip(commands, codes):
            if code:
                raise subprocess.CalledProcessError(code, c)
        subprocess.check_call(link)
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
