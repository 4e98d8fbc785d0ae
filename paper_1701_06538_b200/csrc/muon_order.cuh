// The tiles of a batch's Newton-Schulz products (newton_schulz.cu) in the order in which they are drawn. Plain code of the host and the device: it can be run and looked at without a GPU
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

struct __half;

namespace moe {

constexpr int NS_MAX_SHAPES = 6;
// What a tile is of: A = X X', P = a I + b A + c A A, a product of two of the symmetric matrices, X <- Q X
enum Kind4 { GRAM = 0, POLY = 1, MULT = 2, APPLY = 3 };
// The symmetric matrices
enum { S_A = 0, S_P = 1, S_T = 2, S_P2 = 3, S_Q = 4, SYMMETRIC = 5 };
struct NsShape {
    int32_t rows, cols, ld, M, Mld, first, matrices, left;
    int32_t square, cols3, tiles3;            // tiles of a symmetric matrix (lower half), tiles of X beside each other, of X
    int32_t group, slots;
    int32_t together, turns;                  // steps of a segment; phases of all segments
    const __half *x[2], *s[SYMMETRIC];        // [matrices or slots][rows][ld], [slots][M][Mld]
    float *d;                                 // [SYMMETRIC][slots][M] their diagonals
};
struct NsPlan {
    NsShape s[NS_MAX_SHAPES];
    int32_t shapes, steps, groups, turns;     // turns: of the shape with the most
};

// A segment of n steps as phases, each of which needs all before it: two products at most, a * b -> out. Q of the steps goes from P (or P2) over S_Q to S_T.
struct NsOp { uint8_t kind, a, b, out; };
struct NsPhase { NsOp op[2]; uint8_t n; };
struct NsProgram { NsPhase phase[10]; uint8_t n, squares; };  // squares: products of symmetric matrices, A among them
__host__ __device__ constexpr NsProgram program_of(int steps) {
    constexpr NsOp none = {0, 0, 0, 0}, gram = {GRAM, 0, 0, S_A};
    if (steps == 1) return {{{{gram, none}, 1}, {{{POLY, S_A, S_A, S_P}, none}, 1}, {{{APPLY, S_P, 0, 0}, none}, 1}}, 3, 2};
    if (steps == 2)
        return {{{{gram, none}, 1}, {{{POLY, S_A, S_A, S_P}, none}, 1}, {{{MULT, S_P, S_A, S_T}, none}, 1}, {{{MULT, S_P, S_T, S_A}, none}, 1}, {{{POLY, S_A, S_A, S_P2}, none}, 1},
                 {{{MULT, S_P2, S_P, S_T}, none}, 1}, {{{APPLY, S_T, 0, 0}, none}, 1}}, 7, 6};
    return {{{{gram, none}, 1}, {{{POLY, S_A, S_A, S_P}, none}, 1}, {{{MULT, S_P, S_A, S_T}, none}, 1}, {{{MULT, S_P, S_T, S_A}, none}, 1}, {{{POLY, S_A, S_A, S_P2}, none}, 1},
             {{{MULT, S_P2, S_A, S_T}, {MULT, S_P2, S_P, S_Q}}, 2}, {{{MULT, S_P2, S_T, S_A}, none}, 1}, {{{POLY, S_A, S_A, S_P}, none}, 1}, {{{MULT, S_P, S_Q, S_T}, none}, 1},
             {{{APPLY, S_T, 0, 0}, none}, 1}}, 10, 10};
}
#ifdef __CUDACC__
static __constant__ const NsProgram programs_device[4] = {program_of(1), program_of(1), program_of(2), program_of(3)};
#endif
constexpr NsProgram programs_host[4] = {program_of(1), program_of(1), program_of(2), program_of(3)};
__host__ __device__ __forceinline__ const NsProgram &program(int steps) {
#ifdef __CUDA_ARCH__
    return programs_device[steps];
#else
    return programs_host[steps];
#endif
}
constexpr int MOST_TOGETHER = 3;
constexpr int symmetric_of(int together) { return together == 1 ? 2 : together == 2 ? 4 : 5; }  // that a segment uses, in their order

// Of a matrix of a shape: segments of `together` steps behind one of the rest, if there is one; tiles in all
__host__ __device__ __forceinline__ int32_t turns_of(int32_t steps, int32_t together) {
    const int32_t rest = steps % together;
    return (rest ? program(rest).n : 0) + steps / together * program(together).n;
}
__host__ __device__ __forceinline__ int32_t tiles_of_matrix(const NsShape &h, int32_t steps) {
    const int32_t rest = steps % h.together, full = steps / h.together;
    return (full * program(h.together).squares + (rest ? program(rest).squares : 0)) * h.square + (full + (rest > 0)) * h.tiles3;
}

// {matrix or -1, shape << 16 | segment << 11 | kind << 9 | a << 6 | b << 3 | out, tile's row << 16 | column, slot} of ascending numbers: group of matrices, turn, shape, matrix, tile. A shape's turns are the
// phases of its own segments, one after the other, so that shapes whose segments differ go along with each other
struct NsTileRecord { int32_t matrix, what, place, slot; };
struct NsOrder {
    const NsPlan &p;
    int32_t group, turn, base;   // the group and turn that are at, their first number
    int32_t tiles;               // of them
    int32_t tiles_before;        // of the found one's matrix, in earlier turns
    __host__ __device__ __forceinline__ explicit NsOrder(const NsPlan &p_) : p(p_), group(0), turn(0), base(0), tiles_before(0) { count(); }
    struct At { const NsProgram *g; int32_t segment, phase, squares_before; };  // squares_before: in earlier segments
    __host__ __device__ __forceinline__ At at(const NsShape &h) const {
        const int32_t rest = p.steps % h.together, first = rest ? program(rest).n : 0;
        if (turn < first) return {&program(rest), 0, turn, 0};
        const NsProgram &g = program(h.together);
        const int32_t more = (turn - first) / g.n;
        return {&g, more + (rest > 0), turn - first - more * g.n, (rest ? program(rest).squares : 0) + more * g.squares};
    }
    __host__ __device__ __forceinline__ int32_t here(const NsShape &h) const {
        const int32_t left = h.matrices - group * h.group;
        return left < 0 ? 0 : left < h.group ? left : h.group;
    }
    __host__ __device__ __forceinline__ static int32_t tiles_in(const NsShape &h, const At &a) { return a.phase == a.g->n - 1 ? h.tiles3 : a.g->phase[a.phase].n * h.square; }
    __host__ __device__ __forceinline__ void count() {
        tiles = 0;
        for (int s = 0; s < p.shapes; ++s) {
            const NsShape &h = p.s[s];
            if (turn < h.turns) tiles += here(h) * tiles_in(h, at(h));
        }
    }
    __host__ __device__ __forceinline__ NsTileRecord find(int32_t id) {
        while (group < p.groups && id - base >= tiles) {
            base += tiles;
            if (++turn == p.turns) { turn = 0; ++group; }
            count();
        }
        if (group >= p.groups) return {-1, 0, 0, 0};
        int32_t r = id - base;
        for (int s = 0;; ++s) {
            const NsShape &h = p.s[s];
            if (turn >= h.turns) continue;
            const At a = at(h);
            const int32_t each = tiles_in(h, a), mine = here(h) * each;
            if (r >= mine) { r -= mine; continue; }
            const NsPhase &f = a.g->phase[a.phase];
            const int32_t m = r / each, matrix = group * h.group + m;
            int32_t t = r - m * each, row, col, which = 0, squares_before = a.squares_before;
            if (a.phase == a.g->n - 1) {
                row = t / h.cols3;
                col = t - row * h.cols3;
            } else {
                if (t >= h.square) { t -= h.square; which = 1; }
                for (row = 0; t > row; ++row) t -= row + 1;
                col = t;
            }
            for (int q = 0; q < a.phase; ++q) squares_before += a.g->phase[q].n;
            tiles_before = squares_before * h.square + a.segment * h.tiles3;
            const NsOp &o = f.op[which];
            return {matrix, s << 16 | a.segment << 11 | o.kind << 9 | o.a << 6 | o.b << 3 | o.out, row << 16 | col, matrix % h.slots};
        }
    }
};

}  // namespace moe
