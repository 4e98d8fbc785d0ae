"""The order of the Newton-Schulz products' tiles, compiled for the host: over lists of shapes whose segments differ every tile comes once and behind what it reads, a slot's next user behind its last, and the
phases of a matrix make of x what `steps` times a x + b x^3 + c x^5 does."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1701_06538_b200", "csrc")

HOST = r"""
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <set>
#include <vector>
#include "muon_order.cuh"
using namespace moe;
#define CHECK(ok) do { if (!(ok)) { printf("line %d, list %d\n", __LINE__, list); return 1; } } while (0)
struct Scalar { long tiles; double x[2], s[SYMMETRIC]; };
int main() {
    const double a = 3.4445, b = -4.7750, c = 2.0315;
    long all = 0;
    for (int list = 0; list < 320; ++list) {
        NsPlan p = {};
        p.shapes = 1 + rand() % NS_MAX_SHAPES;
        p.steps = 1 + list % 16;
        const int groups = 1 + rand() % 4;
        long total = 0;
        std::vector<std::vector<Scalar>> m(p.shapes);
        for (int i = 0; i < p.shapes; ++i) {
            NsShape &s = p.s[i];
            const int edge = 1 + rand() % 3, longer = edge + rand() % 3;
            s.square = edge * (edge + 1) / 2; s.cols3 = rand() % 2 ? longer : edge; s.tiles3 = edge * longer;
            s.matrices = 1 + rand() % 20; s.group = (s.matrices + groups - 1) / groups;
            s.slots = s.matrices < 2 * s.group ? s.matrices : 2 * s.group;
            const int together = 1 + rand() % MOST_TOGETHER;
            s.together = p.steps < together ? p.steps : together;
            s.turns = turns_of(p.steps, s.together);
            if (s.turns > p.turns) p.turns = s.turns;
            if ((s.matrices + s.group - 1) / s.group > p.groups) p.groups = (s.matrices + s.group - 1) / s.group;
            total += (long)s.matrices * tiles_of_matrix(s, p.steps);
            for (int k = 0; k < s.matrices; ++k) m[i].push_back({0, {0.05 + 0.9 * rand() / RAND_MAX, NAN}, {NAN, NAN, NAN, NAN, NAN}});
        }
        auto start = m;
        NsOrder order(p), some(p);  // some: as one of several that draw, who does not see every number
        std::set<std::vector<long>> seen;
        for (long id = 0; id < total; ++id) {
            const NsTileRecord t = order.find((int)id);
            CHECK(t.matrix >= 0);
            const int shape = t.what >> 16, segment = t.what >> 11 & 31, kind = t.what >> 9 & 3, from = t.what >> 6 & 7, with = t.what >> 3 & 7, to = t.what & 7, row = t.place >> 16, col = t.place & 0xffff;
            const NsShape &h = p.s[shape];
            Scalar &v = m[shape][t.matrix];
            CHECK(t.slot == t.matrix % h.slots);
            CHECK(v.tiles >= order.tiles_before);
            if (order.tiles_before == 0 && t.matrix >= h.slots) CHECK(m[shape][t.matrix - h.slots].tiles == tiles_of_matrix(h, p.steps));
            CHECK(kind == APPLY ? col < h.cols3 && row * h.cols3 + col < h.tiles3 : col <= row && row * (row + 1) / 2 + col < h.square);
            CHECK(seen.insert({shape, t.matrix, t.what & 0xffff, order.tiles_before, t.place}).second);
            if (row == 0 && col == 0) {
                const double x = v.x[segment & 1];
                if (kind == GRAM) v.s[to] = x * x;
                if (kind == POLY) v.s[to] = a + b * v.s[from] + c * v.s[from] * v.s[with];
                if (kind == MULT) v.s[to] = v.s[from] * v.s[with];
                if (kind == APPLY) v.x[(segment + 1) & 1] = v.s[from] * x;
                if (kind == APPLY) CHECK((segment + 1) * h.together >= p.steps == (v.tiles + h.tiles3 == tiles_of_matrix(h, p.steps)));  // the last segment's
            }
            ++v.tiles;
            ++all;
            if (rand() % 4 == 0) {
                const NsTileRecord u = some.find((int)id);
                CHECK(u.matrix == t.matrix && u.what == t.what && u.place == t.place && some.tiles_before == order.tiles_before);
            }
        }
        CHECK(order.find((int)total).matrix == -1 && order.find((int)total + 1000).matrix == -1 && some.find((int)total).matrix == -1);
        for (int i = 0; i < p.shapes; ++i)
            for (int k = 0; k < p.s[i].matrices; ++k) {
                CHECK(m[i][k].tiles == tiles_of_matrix(p.s[i], p.steps));
                double x = start[i][k].x[0];
                for (int step = 0; step < p.steps; ++step) x = a * x + b * x * x * x + c * x * x * x * x * x;
                const int segments = (p.steps + p.s[i].together - 1) / p.s[i].together;
                CHECK(fabs(m[i][k].x[segments & 1] - x) < 1e-6);  // (64-bit roundings times 6.5 a step at most, seldom above 2)
            }
    }
    printf("%ld tiles\n", all);
    return 0;
}
"""


def test_tiles_come_behind_what_they_read(tmp_path):
    src, exe = tmp_path / "host.cpp", tmp_path / "host"
    src.write_text(HOST)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, "-I", "/usr/local/cuda/include", str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
    assert int(out.stdout.split()[0]) > 500000
