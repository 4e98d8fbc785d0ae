// The matrices of a Muon step's launches, and the launcher of their Newton-Schulz products (newton_schulz.cu)
#pragma once

#include <cuda_fp16.h>

#include "block.cuh"
#include "muon_order.cuh"

namespace moe {

constexpr int MUON_MAX_LIST = 128, MUON_MAX_SHAPES = 6;  // tensors and shapes of a launch (its parameters hold them: 6 KiB, and 1.5 KiB of tensor maps a shape)
constexpr float MUON_UNIT = 1024.0f;                     // what 1 is held as in the products' 16-bit operands
struct MuonEntry {
    void *w, *m;
    const void *g;
    float *master;
    float scale, decay;
    int32_t kind;  // bit 0: bf16 weights, 1: bf16 gradients, 2: bf16 momentum, 3: float masters, 4: weights and masters begin at 32 bytes
};
struct MuonShape {
    int32_t rows, cols, ld;      // ld: elements between rows of the operands, zeros behind the columns
    int32_t first, matrices;     // its matrices are first .. first + matrices - 1
    int32_t chunks, blocks;      // blocks a matrix takes in the first and the second pass
    int32_t chunks_before, blocks_before;  // of the shapes before
    __half *x;                   // [matrices][rows][ld] the updates over their norms, times MUON_UNIT; overwritten
};
// Matrices of up to MUON_MAX_LIST tensors, shape by shape, numbered through
struct MuonBatch {
    MuonEntry t[MUON_MAX_LIST];
    int32_t before[MUON_MAX_LIST + 1];  // matrices of the tensors before
    MuonShape s[MUON_MAX_SHAPES];
    int32_t n, shapes;
    __host__ __device__ __forceinline__ int32_t matrices() const { return before[n]; }
    __device__ __forceinline__ int32_t entry_of(int32_t matrix) const {
        int32_t lo = 0, hi = n;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (before[mid] <= matrix) lo = mid; else hi = mid;
        }
        return lo;
    }
};
static inline int64_t muon_ld(int64_t cols) { return cdiv(cols, 64) * 64; }

struct MuonPasses {
    double *part;     // a sum of squares for every block of the first pass
    int32_t *done;    // [matrices]
    int32_t *next, *status;
    int32_t clear_status, nesterov;
    float momentum, eps, grad_scale;
    const moe_muon_rates *rates;
};

// The whole step by a block a matrix, for small ones (muon_small.cu)
bool muon_is_small(int32_t rows, int32_t cols);
int32_t muon_small_ready();  // whether the device can run it
int32_t launch_muon_small(const MuonBatch &b, const MuonPasses &k, float lr, int32_t steps, cudaStream_t st);

// Newton-Schulz products of a batch's matrices and the step on their weights. Scratch: ns_scratch_bytes
struct NsWork {
    const MuonBatch *batch;
    bool pair;          // see ns_pairs
    int32_t steps;
    int32_t *done;      // [matrices] zeros
    int32_t *next;      // a zero
    int32_t *status;
    void *scratch;
    float lr;
    const moe_muon_rates *rates;  // or nullptr
};
// The launch of them, made before anything of the step is launched: all that may be refused is refused then, and no momentum has taken a step that weights do not take
struct NsMaps { CUtensorMap x_k[2], x_mn[2], s_k[SYMMETRIC], s_mn[SYMMETRIC]; };  // x[0]: all matrices, the others: a ring of slots
struct NsAllMaps { NsMaps m[MUON_MAX_SHAPES]; };
struct NsArgs : NsPlan {
    int32_t *done, *next, *status;
    float lr;
    const moe_muon_rates *rates;
};
static_assert(MUON_MAX_SHAPES == NS_MAX_SHAPES, "shapes of a launch");
struct NsLaunch {
    NsAllMaps maps;
    NsArgs args;
    int64_t tiles;
    bool pair;
};
static inline bool ns_pairs(int32_t rows, int32_t cols) { return imin(rows, cols) > 128; }  // whether a shape takes tiles of SM pairs (768 of 184 x 144: 835 us, by single SMs 1340; 128 of 192 x 448 242 and 342; 64 of 512 x 1024 580 and 712)
int64_t ns_tiles(int32_t rows, int32_t cols, bool pair);                                   // of a matrix, a step
int64_t ns_scratch_bytes(const MuonBatch &batch, bool pair);
int32_t prepare_newton_schulz(const NsWork &w, NsLaunch *to);
int32_t launch_newton_schulz(const NsLaunch &l, const MuonBatch &batch, cudaStream_t st);

}  // namespace moe
