"""The orthogonalisation's rules (csrc/ortho.hip, ortho_gram.hip, host side): what the iteration makes of singular values, which
coefficients the way by X X^T takes, and which way and tiles the sizes take that the GPU tests rely on."""
import os
import subprocess

from test_head_routes import HIPCC, ROOT

BOUNDS = r"""
#include <cstdio>
#include <cstdlib>
#include "ortho_gram.hip"
namespace tppo { int device_compute_units() { return 256; } }
using namespace tppo;
int main() {
    srand48(5);
    int taken = 0, wrong = 0, bounded = 0, tight = 0;
    auto over = [](double x, double most) { return !(x <= most * (1 + 1e-9) + 1e-12); };
    for (int i = 0; i < 60000; ++i) {
        const int all[] = {1, 2, 3, 4, 5, 6, 8, 12, 16}, steps = all[lrand48() % 9];
        const float a = (float)(0.5 + 4.5 * drand48()), b = a * (float)(4 * drand48() - 3), c = i % 5 ? a * (float)(3 * drand48() - 1) : 0.f;
        const NsReach r = ns_reach(steps, a, b, c);
        const bool fits = ns_gram_fits(r, steps, a, b, c);
        taken += fits;
        if (!(r.square < 1e6)) continue;
        ++bounded;
        double largest = 0;
        for (int at = 0; at <= 2000; ++at) {         // singular values as they go
            double l = at / 2000.0, product = 1;
            for (int k = 0; k < steps; ++k) {
                const double m = a + l * (b + l * (double)c);
                product *= fabs(m);
                l *= m * m;
                if (over(product, r.product)) wrong |= 1;
                if (over(fabs(m), r.value)) wrong |= 2;
                if (fabs(m) < r.least * (1 - 1e-9)) wrong |= 4;
                if (over(l, r.square)) wrong |= 8;
                largest = largest > l ? largest : l;
                if (fits && !(l <= 250 && product <= 1000 && fabs(m) <= 250)) wrong |= 16;
            }
        }
        tight += steps > 2 ||                        // (bounds, and not far off)
                 r.square <= 1.02 * (largest > 1 ? largest : 1) + 0.01;
        if (wrong) {
            printf("steps %d a %g b %g c %g: %d\n", steps, a, b, c, wrong);
            break;
        }
    }
    printf("%d\n", wrong);
    printf("%d\n", taken > 2000 && bounded > 20000 && tight > bounded * 0.9);
}
"""

TAKEN = r"""
#include <cstdio>
#include "ortho_gram.hip"
namespace tppo { int device_compute_units() { return 256; } }
int main() {
    const struct { int steps; float a, b, c; } sets[] = {
        // the default, the cubic, two that end in one
        {5, 3.4445f, -4.7750f, 2.0315f}, {1, 3.4445f, -4.7750f, 2.0315f}, {12, 1.5f, -0.5f, 0.f}, {9, 1.875f, -1.25f, 0.375f}, {8, 2.f, -1.5f, 0.5f},
        // more steps than the roundings of pairs allow; a polynomial that comes near zero, or to it, where there are singular values
        {6, 3.4445f, -4.7750f, 2.0315f}, {64, 1.1f, -0.1f, 0.f}, {4, 4.0848f, -6.8946f, 2.9270f}, {5, 3.2556f, -4.9639f, 1.7488f},
        // values that pass what fp16 holds between two points of a grid of 64; a P that shrinks; none
        {5, 1.943f, -4.0259f, 1.0561f}, {8, 2.0255f, -4.4848f, 1.4318f}, {6, 1.6152f, 0.5384f, -0.478f}, {24, 0.4f, 0.f, 0.f}, {0, 3.4445f, -4.7750f, 2.0315f}};
    for (auto& s : sets) printf("%d ", tppo::ns_gram_fits(tppo::ns_reach(s.steps, s.a, s.b, s.c), s.steps, s.a, s.b, s.c));
}
"""

# count, rows, cols, steps: the way (p: pairs, 1: one pass, 3: three), rows of the tiles of X X^T and of B X
SIZES = {(1, 1024, 4096, 5): "p", (1, 1100, 1030, 5): "p", (1, 152064, 192, 5): "p", (1, 152065, 1027, 5): "p", (1, 512, 512, 5): "p",
         (1, 2304, 2304, 5): "1 128 128", (1, 2304, 5120, 5): "1 128 192", (8, 1100, 1030, 5): "1 128 192", (8, 700, 1500, 5): "1 128 160",
         (40, 520, 520, 5): "1 256 128", (16, 530, 700, 5): "1 128 128", (1, 4000, 4090, 5): "1 160 256", (1, 4610, 4520, 5): "1 192 192",
         (1, 5120, 5120, 5): "1 256 256", (1, 5121, 5300, 5): "1 256 256", (1, 5300, 4900, 5): "1 256 256", (1, 152064, 2112, 5): "1 128 256",
         (1, 300, 450, 7): "3 128 128", (1, 700, 511, 10): "3 128 128", (1, 129, 640, 7): "3 128 128", (1, 512, 512, 6): "3 128 128",
         (1, 1024, 1024, 7): "3 128 128", (1, 2304, 2304, 6): "1 128 128", (1, 2304, 2304, 7): "3 128 128"}

WAYS = r"""
#include <cstdio>
#include "ortho_gram.hip"
#include "ortho.hip"
namespace tppo { int device_compute_units() { return 256; } }
using namespace tppo;
int main() {
    long count, rows, cols;
    int steps;
    const float a = 3.4445f, b = -4.7750f, c = 2.0315f;
    const int tile[] = {256, 192, 160, 128};
    for (FILE* f = fopen("SIZES", "r"); fscanf(f, "%ld %ld %ld %d", &count, &rows, &cols, &steps) == 4;) {
        const NsLayout L = ns_layout(count, rows, cols);
        const NsWay way = ns_way(L, count, steps, a, b, c);
        if (way == kNsPairs) puts("p");
        else if (way == kNsThreePasses) puts("3 128 128");
        else printf("1 %d %d\n", tile[ns_shape<true>(L.mp, L.mp, count).shape], tile[ns_shape<false>(L.mp, L.np, count).shape]);
    }
}
"""


def _run(tmp_path, program):
    (tmp_path / "rules.hip").write_text(program)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_15050_amd", "csrc"), str(tmp_path / "rules.hip"),
                    "-o", str(tmp_path / "rules")], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return subprocess.run([str(tmp_path / "rules")], check=True, stdout=subprocess.PIPE, text=True).stdout


def test_no_singular_value_passes_the_bounds(tmp_path):
    assert _run(tmp_path, BOUNDS).split() == ["0", "1"]


def test_coefficients_of_the_way_by_pairs(tmp_path):
    assert _run(tmp_path, TAKEN).split() == ["1"] * 5 + ["0"] * 9


def test_ways_and_tiles(tmp_path):
    (tmp_path / "sizes").write_text("\n".join(" ".join(map(str, size)) for size in SIZES))
    got = _run(tmp_path, WAYS.replace("SIZES", str(tmp_path / "sizes"))).splitlines()
    assert dict(zip(SIZES, got)) == SIZES
