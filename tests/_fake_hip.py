"""The library on a stand-in for the HIP runtime (csrc/fake_hip.cpp): what it asks
of the runtime, call by call, without a GPU.  A script runs in a process of its own,
where the stand-in is loaded before the library, and prints a JSON value."""
import ctypes
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCE = os.path.join(HERE, "csrc", "fake_hip.cpp")


def build(folder) -> str:
    out = os.path.join(str(folder), "libfake_hip.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", SOURCE, "-o", out], check=True)
    return out


def run(fake: str, script: str):
    """The value that `script` leaves in `result`."""
    program = ("import sys; sys.path.insert(0, %r)\nfrom _fake_hip import Library\nL = Library(%r)\n%s\n"
               "import json; print(json.dumps(result))" % (HERE, fake, script))
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout.splitlines()[-1])


P, I32, I64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
X = 0x7000_0000_0000        # stands for the caller's device memory, 16-byte aligned


class Library:
    """The entry points, and the stand-in's log."""

    def __init__(self, fake: str):
        self.fake = ctypes.CDLL(fake, mode=ctypes.RTLD_GLOBAL)
        self.fake.fake_log.restype = self.fake.fake_kernels.restype = ctypes.c_char_p
        self.fake.fake_held.restype = ctypes.c_size_t
        self.fake.fake_room.argtypes = [ctypes.c_size_t]
        self.fake.fake_capture.argtypes = [P, ctypes.c_ulonglong]
        self.fake.fake_fail.argtypes = [ctypes.c_char_p, I32]
        self.emu = ctypes.CDLL(os.path.join(HERE, "..", "paper_2609_04663_amd", "libemu.so"))
        self.emu.emu_set_stream.argtypes = [P]
        self.emu.emu_last_error.restype = ctypes.c_char_p
        self.emu.emu_workspace_bytes.restype = I64

    def log(self, plans=False):
        """The lines since the last call, as lists of words and numbers; a launch
        is ["launch", stream, x, y, z, threads, kernel].  With plans, those of 4-bit
        products: ["plan", waves along the reduction, passes, splits]."""
        lines = []
        for line in self.fake.fake_log().decode().splitlines():
            if line.startswith("plan") and not plans:
                continue
            words = line.split(" ", 6) if line.startswith("launch") else line.split(" ")
            lines.append([int(w) if w.lstrip("-").isdigit() else w for w in words])
        self.fake.fake_clear()
        return lines

    def kernels(self):
        """The kernels launched since the last look at the log."""
        return [short(line[6]) for line in self.log() if line[0] == "launch"]

    def all_kernels(self):
        return sorted(short(k) for k in self.fake.fake_kernels().decode().splitlines())

    def stream(self, s):
        return self.emu.emu_set_stream(s)

    # calls with the least that a test has to say; leading dimensions as the rows' lengths
    def sgemm(self, M=64, N=64, K=64):
        return self.emu.emu_sgemm(I64(M), I64(N), I64(K), P(X), I64(K), P(X), I64(N), P(X), I64(N))

    def route(self, dtype=0, T=100, E=64, k=8, scope=0):
        return self.emu.emu_moe_route(dtype, I64(T), E, k, scope, P(X), I64(E), P(X), P(X), P(X), P(X), P(X))

    def grouped(self, dtype, transb, E, R, N, K, rows=False, XR=None, x=X, ldx=None, w=X, ldw=None, stride=None):
        ldw = ldw or (K if transb == "T" else N)
        stride = ldw * (N if transb == "T" else K) if stride is None else stride
        return self.emu.emu_grouped_gemm(dtype, ctypes.c_char(transb.encode()), E, I64(R), I64(N), I64(K), P(x),
                                         I64(ldx or K), I64(R if XR is None else XR), P(X) if rows else None,
                                         P(w), I64(ldw), I64(stride), P(X), P(X), I64(N))

    def wgrad(self, dtype, transb, E, R, N, K, rows=False, XR=None, x=X, ldx=None, dy=X, lddy=None):
        ldw = K if transb == "T" else N
        return self.emu.emu_grouped_wgrad(dtype, ctypes.c_char(transb.encode()), E, I64(R), I64(N), I64(K), P(x),
                                          I64(ldx or K), I64(R if XR is None else XR), P(X) if rows else None,
                                          P(dy), I64(lddy or N), P(X), P(X), I64(ldw),
                                          I64(ldw * (N if transb == "T" else K)))

    def q4(self, dtype, E, R, N, K, group=64, mins=False, rows=False, XR=None, x=X):
        return self.emu.emu_q4_gemm(dtype, E, I64(R), I64(N), I64(K), group, P(x), I64(K),
                                    I64(R if XR is None else XR), P(X) if rows else None, P(X), P(X),
                                    P(X) if mins else None, P(X) if E != 1 else None, P(X), I64(N))


def short(kernel: str) -> str:
    """A kernel's name and template arguments, without namespaces and parameters."""
    name = kernel.replace("(anonymous namespace)::", "").replace("emu::", "")
    name = name[5:] if name.startswith("void ") else name
    name = name.replace("<signed char", "<bf16").replace("<unsigned char", "<f16")
    depth = 0
    for i, c in enumerate(name):
        depth += (c == "<") - (c == ">")
        if c == "(" and depth == 0:
            return name[:i]
    return name
