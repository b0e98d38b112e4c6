"""The group norm's plan (csrc/group_norm.cuh) on the host alone: a small program
made of the library's own header answers which kernels a shape gets on 152 SMs,
in a process of its own, without a GPU."""
import collections
import os
import subprocess

from paper_2003_04296_gb300 import build as libbuild

PROGRAM = r"""
#include <stdio.h>
#include "group_norm.cuh"
namespace minw_host {
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int num_sms() { return 152; }
bool pdl_enabled() { return false; }
bool allow_shared(const void *, int) { return false; }
void max_shared_carveout(const void *) {}
}
int main() {
    using namespace minw::gn;
    int B, P, C, G, xb, yb, backward, off;
    long long ld;
    while (scanf("%d %d %d %d %lld %d %d %d %d", &B, &P, &C, &G, &ld, &off, &xb, &yb, &backward) == 9) {
        const int xt = xb == 2 ? MINW_BF16 : MINW_F32, yt = yb == 2 ? MINW_BF16 : MINW_F32;
        const void *x = reinterpret_cast<const void *>(4096 + (uintptr_t)(off * xb));
        const void *y = reinterpret_cast<const void *>(4096 + (uintptr_t)(off * yb));
        int V = xb == 2 && yb == 2 ? 8 : 4;
        while (V > 1 && (C % V != 0 || !fits(x, ld, xt, V) || !fits(y, ld, yt, V))) V = V == 8 ? 4 : 1;
        Args a{};
        a.B = B; a.P = P; a.C = C; a.G = G; a.Cg = C / G; a.ldx = ld;
        Plan pl{};
        const char *ways[] = {"shared", "held", "reread", "chunks"};
        const bool one = plan(a, pl, xb, backward ? yb : 0, V);
        printf("%s %d %d %d %d %d %d %d %d %d %d\n", one ? ways[pl.way] : "stream", one ? pl.V : V, pl.GPT, pl.smem, a.L,
               a.slabs, a.rows, a.groups, a.chunks, a.ppc, a.per);
        fflush(stdout);
    }
    return 0;
}
"""

Plan = collections.namedtuple("Plan", "way V GPT smem L slabs rows groups cluster ppc per")


def compiled(folder):
    """The program's path."""
    src, exe = os.path.join(folder, "plan.cu"), os.path.join(folder, "plan")
    with open(src, "w") as f:
        f.write(PROGRAM)
    cmd = [libbuild.NVCC, *libbuild.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I",
           os.path.join(libbuild.ROOT, "include"), "-I", libbuild.CSRC, src, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed:\n{r.stderr}")
    return exe


def plans(exe, shapes):
    """A Plan for each of the shapes (B, P, C, G, row length, first channel, type of x, type of y or dy, backward), types
    "f" or "b"; a program that ends early fails with the shape it ended at."""
    size = {"f": 4, "b": 2}
    text = "".join(f"{B} {P} {C} {G} {ld} {off} {size[tx]} {size[ty]} {int(back)}\n"
                   for B, P, C, G, ld, off, tx, ty, back in shapes)
    r = subprocess.run([exe], input=text, capture_output=True, text=True)
    lines = r.stdout.splitlines()
    if r.returncode != 0 or len(lines) != len(shapes):
        raise AssertionError(f"no plan (status {r.returncode}) for {shapes[len(lines)]}")
    return [Plan(w[0], *map(int, w[1:])) for w in map(str.split, lines)]
