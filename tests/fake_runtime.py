"""The library's launches without a GPU: its calls into the HIP runtime end in a stand-in that takes down what is launched.

A child process loads the stand-in for all to see, then libgspc.so, whose symbols it serves, and makes the calls.  A launch of 2^32
threads and more is refused, as the runtime does."""
import json
import subprocess
import sys

from paper_2006_09791_amd import binding as b

RUNTIME = r"""
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim3;
static struct { dim3 grid, block; size_t lds; void *stream; } config;
static int last;
static const void *stubs[1 << 16];
static const char *names[1 << 16];
static int known;
void (*take_down)(const char *, unsigned, unsigned, void **);

void **__hipRegisterFatBinary(const void *p) { static void *handle; (void)p; return &handle; }
void __hipUnregisterFatBinary(void **p) { (void)p; }
void __hipRegisterFunction(void **m, const void *stub, char *device, const char *name, unsigned n, void *a, void *b, void *c, void *d, int *e) {
    (void)m, (void)device, (void)n, (void)a, (void)b, (void)c, (void)d, (void)e;
    if (known < 1 << 16) stubs[known] = stub, names[known++] = name;
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, void *stream) {
    config.grid = grid, config.block = block, config.lds = lds, config.stream = stream;
    return 0;
}
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, void **stream) {
    *grid = config.grid, *block = config.block, *lds = config.lds, *stream = config.stream;
    return 0;
}
int hipLaunchKernel(const void *stub, dim3 grid, dim3 block, void **args, size_t lds, void *stream) {
    (void)lds, (void)stream;
    if (grid.x == 0 || grid.y != 1 || grid.z != 1 || (unsigned long long)grid.x * block.x > 0xffffffffull) return last = 9;
    for (int i = 0; i < known; ++i)
        if (stubs[i] == stub) take_down(names[i], grid.x, block.x, args);
    return 0;
}
int hipGetLastError(void) { const int e = last; last = 0; return e; }
const char *hipGetErrorString(int e) { (void)e; return "refused"; }
int hipFuncSetAttribute(const void *f, int a, int v) { (void)f, (void)a, (void)v; return 0; }
"""

CHILD = r"""
import ctypes, json, re, sys
runtime, library = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL), None
launches, decode = [], {}

def take_down(name, blocks, threads, args):
    short = re.match(r"_ZN4gspc(\d+)(\w+)", name.decode())
    short = short[2][:int(short[1])]
    values = [(name if i < 0 else bytes((ctypes.c_char * size).from_address(args[i]))).hex() for i, size in decode.get(short, [])]
    launches.append([short, blocks, threads, values])
kind = ctypes.CFUNCTYPE(None, ctypes.c_char_p, ctypes.c_uint, ctypes.c_uint, ctypes.POINTER(ctypes.c_void_p))
keep = kind(take_down)
ctypes.c_void_p.in_dll(runtime, "take_down").value = ctypes.cast(keep, ctypes.c_void_p).value
library = ctypes.CDLL(sys.argv[2])
types = {t._type_: t for t in (ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float)}
work, out = json.load(sys.stdin), []
decode.update(work["decode"])
for name, codes, result, args in work["calls"]:
    call = getattr(library, name)
    call.argtypes, call.restype = [types[c] for c in codes], types[result]
    del launches[:]
    rc = call(*args)
    out.append([rc, list(launches)])
json.dump(out, sys.stdout)
"""


def build(folder):
    """The stand-in, compiled into `folder`."""
    (folder / "runtime.c").write_text(RUNTIME)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", str(folder / "runtime.c"), "-o", str(folder / "runtime.so")], check=True)
    return str(folder / "runtime.so")


def launches(runtime, calls, decode):
    """[(result, [(kernel, blocks, threads of a block, arguments)])] for calls [(entry point, arguments)]: of each kernel those arguments
    that `decode` names as (number, bytes), raw; number -1 is the kernel's whole name."""
    lib = b.load()
    work = [(name, [t._type_ for t in getattr(lib, name).argtypes], getattr(lib, name).restype._type_, args) for name, args in calls]
    r = subprocess.run([sys.executable, "-c", CHILD, runtime, b.LIB_PATH], input=json.dumps({"calls": work, "decode": decode}), capture_output=True,
                       text=True, check=False, timeout=100)
    assert r.returncode == 0, r.stderr
    return [(rc, [(k, blocks, threads, [bytes.fromhex(v) for v in args]) for k, blocks, threads, args in found]) for rc, found in json.loads(r.stdout)]
