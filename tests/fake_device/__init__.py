"""The operators' argument checks without a GPU, on addresses that count as device
memory (fake_device.c): refusals that look at memory, and calls that are let through."""
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(os.path.dirname(HERE)), "paper_2607_18957_amd", "libii.so")

# in a process of its own, where the runtime's functions come from here first
_CHILD = """
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
for name, args in json.load(sys.stdin):
    f = getattr(lib, name)
    f.argtypes = [ctypes.c_char_p] * len(args) + [ctypes.c_void_p]
    print(f(*[None if a is None else bytes.fromhex(a) for a in args], None))
"""


def build(to: str) -> str:
    """The runtime as a library in the folder `to`."""
    lib = os.path.join(to, "fake_device.so")
    subprocess.check_call(["gcc", "-std=c11", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", "-o", lib, os.path.join(HERE, "fake_device.c")])
    return lib


def codes(fake: str, calls) -> list[int]:
    """What each call (name, arguments but the stream as bytes or None) returns."""
    sent = json.dumps([(n, [None if a is None else a.hex() for a in args]) for n, args in calls])
    r = subprocess.run([sys.executable, "-c", _CHILD, fake, LIB], input=sent, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return [int(x) for x in r.stdout.split()]
