"""The library's host side over a CUDA runtime and kernels that only note what they are asked for (fake_device.cpp)."""
import concurrent.futures as cf
import ctypes
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2107_06960_gb300", "csrc")
SOURCES = ["attention.cpp", "decode.cpp", "runtime.cpp", "planner.cpp", "order.cpp", "noalloc.cu"]


class Fake:
    """The entry points over the fake, by the binding's signatures; notes(): what was asked for since the last reset."""

    def __init__(self, mf, path):
        self.lib = ctypes.CDLL(path)
        for name, res, args in mf._SIGNATURES:
            f = getattr(self.lib, name, None)
            if f is not None:
                f.restype, f.argtypes = res, args
        self.lib.fake_notes.restype = ctypes.c_char_p
        self.lib.fake_fail.argtypes = [ctypes.c_char_p]

    def notes(self):
        return self.lib.fake_notes().decode().splitlines()

    def reset(self):
        self.lib.fake_reset()

    def fail(self, name):
        self.lib.fake_fail(name.encode())


def build(mf, folder):
    include = []
    for d in (os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"), CSRC, os.path.join(ROOT, "include")):
        include += ["-I", d]

    def compile_(src):
        obj = os.path.join(folder, os.path.basename(src) + ".o")
        subprocess.run(["g++", "-std=c++17", "-O0", "-fPIC"] + include + ["-x", "c++", "-c", src, "-o", obj], check=True)
        return obj
    files = [os.path.join(CSRC, s) for s in SOURCES] + [os.path.join(HERE, "fake_device.cpp")]
    with cf.ThreadPoolExecutor(max_workers=len(files)) as ex:
        objs = list(ex.map(compile_, files))
    path = os.path.join(folder, "libfake.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic"] + objs + ["-o", path], check=True)
    return Fake(mf, path)
