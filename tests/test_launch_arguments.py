"""What the kernels of relpos.h's window form are handed follows from the call alone, not from what the stack held before it.

In a process of its own, in which a launch keeps the first bytes of the kernel's arguments and does nothing else (no GPU is used).
"""
import subprocess
import sys

from paper_2409_06206_amd import build, relpos

SHIM = """
#include <string.h>
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim3;
static unsigned char seen[4096];
static size_t keep;
static int launches;
void keep_bytes(size_t bytes) { keep = bytes; }
const unsigned char *kept(void) { return seen; }
int count(void) { return launches; }
static dim3 grid, block;
static size_t shared;
static void *stream;
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, void *t) { grid = g; block = b; shared = s; stream = t; return 0; }
int __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *s, void **t) { *g = grid; *b = block; *s = shared; *t = stream; return 0; }
int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **args, size_t s, void *t) { ++launches; memcpy(seen, args[0], keep); return 0; }
int hipGetLastError(void) { return 0; }
"""

# (Args of csrc/relpos.hip: five pointers, a long, fifteen numbers, the edges)
BYTES = 5 * 8 + 8 + 15 * 4 + 127 * 4

CHILD = """
import ctypes, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
shim.kept.restype = ctypes.c_void_p
shim.keep_bytes.argtypes = [ctypes.c_size_t]
shim.keep_bytes(int(sys.argv[3]))
for name, n in (("relpos_forward", 4), ("relpos_backward", 5)):
    getattr(lib, name).argtypes = [ctypes.c_void_p] * n
window, others = bytes.fromhex(sys.argv[4]), [bytes.fromhex(a) for a in sys.argv[5:]]
for pass_ in ("forward", "backward"):
    seen = set()
    for other in others:
        for desc, ws in ((other, 1 << 40), (window, None)):
            before = shim.count()
            status = lib.relpos_forward(desc, 1 << 30, 1 << 34, None) if pass_ == "forward" else lib.relpos_backward(desc, 1 << 34, 1 << 30, ws, None)
            assert status == 0 and shim.count() > before, (pass_, status)
        seen.add(ctypes.string_at(shim.kept(), int(sys.argv[3])))
    print(pass_, len(seen))
"""


def test_arguments_of_a_window_are_the_same_bytes_every_call(tmp_path):
    source, shim = tmp_path / "shim.c", tmp_path / "shim.so"
    source.write_text(SHIM)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(shim), str(source)], check=True)
    window = relpos.make_desc(6, [1, 2, 4], "bf16", relpos.RELPOS_BIDIRECTIONAL, window=8)
    # sequences of other tiles, whose plans leave other values where a window's plan will lie
    others = [relpos.make_desc(6, [1, 2, 4], "bf16", 0, q, k, batch=2) for q, k in ((5, 4000), (4000, 4000), (130, 7), (2000, 513))]
    out = subprocess.run([sys.executable, "-c", CHILD, str(shim), build.LIB_PATH, str(BYTES), *(bytes(d).hex() for d in (window, *others))],
                         check=True, capture_output=True, text=True, timeout=60).stdout
    assert out.split() == ["forward", "1", "backward", "1"], out
