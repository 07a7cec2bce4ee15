"""What the library launches, seen from the host: calls in a child process in which hipLaunchKernel writes down its grid and launches nothing (a few lines of C that are preloaded),
so that sizes can be asked for that no test could hold.  Needs no GPU and touches none."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <stddef.h>
#include <stdio.h>
typedef struct { unsigned x, y, z; } dims;
static dims grid, block;
static size_t lds;
int __hipPushCallConfiguration(dims g, dims b, size_t bytes, void *stream) { grid = g; block = b; lds = bytes; return 0; }
int __hipPopCallConfiguration(dims *g, dims *b, size_t *bytes, void **stream) { *g = grid; *b = block; *bytes = lds; *stream = NULL; return 0; }
int hipGetLastError(void) { return 0; }
int hipLaunchKernel(const void *f, dims g, dims b, void **args, size_t bytes, void *stream)
{
    printf("launch %u %u %u %u %u %u %zu\n", g.x, g.y, g.z, b.x, b.y, b.z, bytes);
    fflush(stdout);
    return 0;
}
"""


def build(folder):
    src, lib = os.path.join(str(folder), "record.c"), os.path.join(str(folder), "librecord.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-o", lib, src])
    return lib


def launches(lib, call):
    """[(grid, block, bytes of LDS)] of the launches that `call`, Python with the package as P, makes."""
    env = dict(os.environ, PYTHONPATH=ROOT)
    env["LD_PRELOAD"] = lib + ((":" + env["LD_PRELOAD"]) if env.get("LD_PRELOAD") else "")
    r = subprocess.run([sys.executable, "-c", "import paper_1812_07625_amd as P\n" + call], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    rows = [[int(w) for w in line.split()[1:]] for line in r.stdout.splitlines() if line.startswith("launch ")]
    return [(tuple(a[:3]), tuple(a[3:6]), a[6]) for a in rows]
