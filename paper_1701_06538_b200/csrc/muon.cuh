// The Muon step's matrices of one shape, and the launcher of their Newton-Schulz products (newton_schulz.cu)
#pragma once

#include <cuda_fp16.h>

#include "block.cuh"

namespace moe {

constexpr int MUON_MAX_LIST = 64;           // tensors of a launch (a launch's parameters hold them: 3 KiB)
constexpr float MUON_UNIT = 1024.0f;        // what 1 is held as in the products' 16-bit operands
struct MuonEntry {
    void *w, *m;
    const void *g;
    float *master;
    float scale, decay;
    int32_t kind;  // bit 0: bf16 weights, 1: bf16 gradients, 2: bf16 momentum, 3: float masters
};
// Matrices [rows, cols] of up to MUON_MAX_LIST tensors, numbered through
struct MuonBatch {
    MuonEntry t[MUON_MAX_LIST];
    int32_t first[MUON_MAX_LIST + 1];  // matrices of the tensors before
    int32_t n, rows, cols;
    __device__ __forceinline__ int32_t entry_of(int32_t matrix) const {
        int32_t lo = 0, hi = n;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (first[mid] <= matrix) lo = mid; else hi = mid;
        }
        return lo;
    }
};
static inline int64_t muon_ld(int64_t cols) { return cdiv(cols, 64) * 64; }  // elements between rows of the operands, zeros behind the columns

// Newton-Schulz products of a batch's matrices and the step on their weights. Scratch: ns_scratch_bytes behind 256 bytes
struct NsWork {
    const MuonBatch *batch;
    int32_t matrices, steps;
    __half *x;          // [matrices][rows][ld] the updates over their norms, times MUON_UNIT; overwritten
    int32_t *done;      // [matrices] zeros
    int32_t *next;      // a zero
    int32_t *status;
    void *scratch;
    float lr;
    const moe_muon_rates *rates;  // or nullptr
};
int64_t ns_scratch_bytes(int32_t rows, int32_t cols, int64_t matrices);
int32_t launch_newton_schulz(const NsWork &w, cudaStream_t st);

}  // namespace moe
