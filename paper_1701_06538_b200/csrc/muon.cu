// The Muon step (Jordan et al., 2024) over a list of batches of matrices: momentum, the update orthogonalised by Newton-Schulz products, weights. For every matrix
//   m = momentum m + g,   u = g + momentum m  (or m),   X = u / (|u| + eps)  over its Frobenius norm,   then newton_schulz.cu
// Here: the two passes before the products, both bound by memory. The first makes m and the sums of u's squares, the second X, which needs the whole matrix' norm. u is made of the
// momentum as it is held, so that the second pass makes the same one again.
#include <float.h>

#include <memory>
#include <vector>

#include "muon.cuh"
#include "muon_passes.cuh"
#include "pairs.cuh"
#include "tc.cuh"
#include "vectors.cuh"

namespace moe {

namespace {

constexpr int THREADS = PASS_THREADS, WARPS = THREADS / 32, CHUNK = THREADS * EACH * TURNS;  // CHUNK: of the second pass
constexpr int64_t MOST_X = (int64_t)1 << 30;   // bytes of X of a launch (one matrix at least)

__device__ __forceinline__ double sum_of_block(double v, double *sh) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += sh[w];
    return s;
}

__global__ void __launch_bounds__(THREADS) muon_momentum_kernel(const __grid_constant__ MuonBatch b, const MuonPasses k) {
    __shared__ double sh[WARPS];
    wait_previous_kernel();
    int q = 0;
    while (q + 1 < b.shapes && (int32_t)blockIdx.x >= b.s[q + 1].chunks_before) ++q;
    const MuonShape &s = b.s[q];
    const int32_t here = (int32_t)blockIdx.x - s.chunks_before, in_shape = here / s.chunks, chunk = here - in_shape * s.chunks, matrix = s.first + in_shape;
    if (threadIdx.x == 0 && chunk == 0) {
        k.done[matrix] = 0;
        if (matrix == 0) {
            *k.next = 0;
            if (k.clear_status) *k.status = 0;
        }
    }
    const int32_t i = b.entry_of(matrix);
    const int64_t each = (int64_t)s.rows * s.cols, first = (matrix - b.before[i]) * each, at = first + (int64_t)chunk * PASS_CHUNK, end = min(at + PASS_CHUNK, first + each);
    const float grad_scale = k.rates ? k.rates->grad_scale : k.grad_scale;
    // vectors of eight where every matrix begins at one
    double v = each % EACH == 0 ? momentum_block<true>(b.t[i], at, end, grad_scale, k) : momentum_block<false>(b.t[i], at, end, grad_scale, k);
    v = sum_of_block(v, sh);
    if (threadIdx.x == 0) k.part[blockIdx.x] = v;
}

// X in rows of ld elements, zeros behind the columns: a block has CHUNK of them, a piece of eight a thread at a time
template <typename GT, typename MT, bool VECTORS>
__device__ __forceinline__ void normalise_chunk(const GT *g, const MT *m, int64_t first, __half *x, int64_t begin, int64_t pieces, int32_t cols, int32_t ld, float grad_scale, const Factor &by,
                                                const MuonPasses &k) {
    const int32_t in_row = ld / EACH;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int64_t piece = begin + i * THREADS + threadIdx.x;
        if (piece >= pieces) break;
        const int32_t row = (int32_t)((uint32_t)piece / (uint32_t)in_row), col = ((int32_t)piece - row * in_row) * EACH, live = cols - col;
        uint32_t out[EACH / 2] = {0u, 0u, 0u, 0u};
        if (live > 0) {
            const int64_t at = first + (int64_t)row * cols + col;
            float gv[EACH], mv[EACH];
            load8<MT, VECTORS>(m, at, live, mv);
            if (k.nesterov) load8<GT, VECTORS>(g, at, live, gv);
#pragma unroll
            for (int j = 0; j < EACH; j += 2) {
                float u[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) u[q] = by(k.nesterov ? fmaf(k.momentum, mv[j + q], gv[j + q] * grad_scale) : mv[j + q]);
                const __half2 h = __floats2half2_rn(u[0], u[1]);
                out[j / 2] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        *reinterpret_cast<uint4 *>(x + piece * EACH) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}
template <bool VECTORS>
__device__ __forceinline__ void normalise_block(const MuonEntry &t, const MuonShape &s, int64_t first, __half *x, int64_t begin, float grad_scale, const Factor &by, const MuonPasses &k) {
    const int64_t pieces = (int64_t)s.rows * (s.ld / EACH);
    switch (t.kind & 6) {
        case 0: return normalise_chunk<float, float, VECTORS>(static_cast<const float *>(t.g), static_cast<const float *>(t.m), first, x, begin, pieces, s.cols, s.ld, grad_scale, by, k);
        case 2: return normalise_chunk<bf16, float, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<const float *>(t.m), first, x, begin, pieces, s.cols, s.ld, grad_scale, by, k);
        case 4: return normalise_chunk<float, bf16, VECTORS>(static_cast<const float *>(t.g), static_cast<const bf16 *>(t.m), first, x, begin, pieces, s.cols, s.ld, grad_scale, by, k);
        default: return normalise_chunk<bf16, bf16, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<const bf16 *>(t.m), first, x, begin, pieces, s.cols, s.ld, grad_scale, by, k);
    }
}
__global__ void __launch_bounds__(THREADS) muon_normalise_kernel(const __grid_constant__ MuonBatch b, const MuonPasses k) {
    __shared__ double sh[WARPS];
    wait_previous_kernel();
    // Backwards: what the first pass has touched last is in L2 still, and so is what the products read first
    const int32_t id = (int32_t)(gridDim.x - 1 - blockIdx.x);
    int q = 0;
    while (q + 1 < b.shapes && id >= b.s[q + 1].blocks_before) ++q;
    const MuonShape &s = b.s[q];
    const int32_t here = id - s.blocks_before, in_shape = here / s.blocks, block = here - in_shape * s.blocks, matrix = s.first + in_shape;
    double v = 0.0;
    for (int32_t c = threadIdx.x; c < s.chunks; c += THREADS) v += k.part[s.chunks_before + (int64_t)in_shape * s.chunks + c];
    const Factor by(sqrt(sum_of_block(v, sh)) + (double)k.eps);
    const int32_t i = b.entry_of(matrix);
    const int64_t first = (int64_t)(matrix - b.before[i]) * s.rows * s.cols, begin = (int64_t)block * (CHUNK / EACH);
    __half *x = s.x + (int64_t)in_shape * s.rows * s.ld;
    const float grad_scale = k.rates ? k.rates->grad_scale : k.grad_scale;
    // vectors of eight where every row begins at one
    if (s.cols % EACH == 0) normalise_block<true>(b.t[i], s, first, x, begin, grad_scale, by, k);
    else normalise_block<false>(b.t[i], s, first, x, begin, grad_scale, by, k);
}

bool starts_at(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
int32_t check_tensor(const moe_muon_tensor &t) {
    if (t.count < 0 || t.count > (int64_t)1 << 24 || t.rows <= 0 || t.cols <= 0 || t.rows > MOE_MUON_MAX_SIDE || t.cols > MOE_MUON_MAX_SIDE) return MOE_ERR_INVALID_ARG;
    for (int32_t type : {t.w_type, t.g_type, t.m_type})
        if (type != MOE_F32 && type != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (!(t.weight_decay >= 0.0f) || !(t.weight_decay <= FLT_MAX) || !(fabsf(t.scale) <= FLT_MAX)) return MOE_ERR_INVALID_ARG;
    if (t.count == 0) return MOE_OK;
    const void *all[] = {t.w, t.g, t.m};
    for (const void *p : all)
        if (!p || !starts_at(p, 16)) return MOE_ERR_INVALID_ARG;
    if (t.master && (t.w_type != MOE_BF16 || !starts_at(t.master, 16))) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

// The list's shapes, each with its tensors in the list's order
struct Shape {
    int32_t rows, cols;
    int64_t matrices;
    std::vector<int32_t> tensors;
    int64_t x_bytes() const { return matrices * rows * muon_ld(cols) * 2; }
};
// Matrices from * matrices / parts on, up to those of the next part, of every shape; false: more tensors than a launch takes
bool fill_batch(const moe_muon_tensor *tensors, const Shape *const *shapes, int n, int64_t part, int64_t parts, MuonBatch *b) {
    b->n = b->shapes = b->before[0] = 0;
    int64_t chunks = 0, blocks = 0;
    for (int q = 0; q < n; ++q) {
        const Shape &h = *shapes[q];
        const int64_t from = h.matrices * part / parts, to = h.matrices * (part + 1) / parts, each = (int64_t)h.rows * h.cols;
        if (from == to) continue;
        MuonShape &s = b->s[b->shapes++];
        s.rows = h.rows; s.cols = h.cols; s.ld = (int32_t)muon_ld(h.cols);
        s.first = b->before[b->n]; s.matrices = (int32_t)(to - from);
        s.chunks = (int32_t)cdiv(each, PASS_CHUNK); s.blocks = (int32_t)cdiv((int64_t)s.rows * s.ld, CHUNK);
        s.chunks_before = (int32_t)chunks; s.blocks_before = (int32_t)blocks;
        s.x = nullptr;
        chunks += (to - from) * s.chunks; blocks += (to - from) * s.blocks;
        if (chunks > INT32_MAX || blocks > INT32_MAX) return false;
        int64_t at = 0;
        for (int32_t i : h.tensors) {
            const moe_muon_tensor &t = tensors[i];
            const int64_t a = imax(from, at), z = imin(to, at + t.count);
            if (a < z) {
                if (b->n == MUON_MAX_LIST) return false;
                auto on = [&](const void *p, int32_t type) { return static_cast<char *>(const_cast<void *>(p)) + (a - at) * each * (int64_t)act_bytes(type); };
                MuonEntry &e = b->t[b->n];
                e.w = on(t.w, t.w_type); e.g = on(t.g, t.g_type); e.m = on(t.m, t.m_type);
                e.master = t.master ? t.master + (a - at) * each : nullptr;
                e.scale = t.scale; e.decay = t.weight_decay;
                e.kind = (t.w_type == MOE_BF16 ? 1 : 0) | (t.g_type == MOE_BF16 ? 2 : 0) | (t.m_type == MOE_BF16 ? 4 : 0) | (t.master ? 8 : 0) | (starts_at(t.w, 32) && starts_at(t.master, 32) ? 16 : 0);
                b->before[b->n + 1] = b->before[b->n] + (int32_t)(z - a);
                ++b->n;
            }
            at += t.count;
        }
    }
    return true;
}
// The list in launches; `run` is given each. Shapes that fill the tiles of SM pairs go together, those that one block does from beginning to end, and the others. Where there are SM pairs'
// tiles and these are an eighth of them or less, they go along: the chain of a gate's products then runs beside the experts' (32 experts of 512 x 1024 and their gate 576 us, the gate by itself
// afterwards 624; 16 of 256 x 512 171 and 213).
enum How { SMALL = 0, SINGLE = 1, PAIRS = 2 };
template <typename Run> int32_t for_each_launch(const moe_muon_tensor *tensors, int32_t count, Run run) try {
    std::vector<Shape> all;
    for (int32_t i = 0; i < count; ++i) {
        const moe_muon_tensor &t = tensors[i];
        if (t.count == 0) continue;
        size_t q = 0;
        while (q < all.size() && (all[q].rows != t.rows || all[q].cols != t.cols)) ++q;
        if (q == all.size()) all.push_back({t.rows, t.cols, 0, {}});
        all[q].matrices += t.count;
        all[q].tensors.push_back(i);
    }
    std::vector<const Shape *> kinds[3];
    int64_t others = 0, paired = 0;
    size_t shapes_of_all = 0;
    for (const Shape &s : all) {
        const How how = ns_pairs(s.rows, s.cols) ? PAIRS : muon_is_small(s.rows, s.cols) ? SMALL : SINGLE;
        kinds[how].push_back(&s);
        (how == PAIRS ? paired : others) += s.matrices * ns_tiles(s.rows, s.cols, true);
        ++shapes_of_all;
    }
    if (others * 8 <= paired && shapes_of_all <= (size_t)MUON_MAX_SHAPES)
        for (int how = SMALL; how < PAIRS; ++how) {
            kinds[PAIRS].insert(kinds[PAIRS].end(), kinds[how].begin(), kinds[how].end());
            kinds[how].clear();
        }
    MuonBatch b;
    for (int how = PAIRS; how >= SMALL; --how)
        for (size_t from = 0; from < kinds[how].size(); from += MUON_MAX_SHAPES) {
            const Shape *const *shapes = kinds[how].data() + from;
            const int n = (int)imin(MUON_MAX_SHAPES, (int64_t)(kinds[how].size() - from));
            int64_t bytes = 1, most = 0;
            for (int q = 0; q < n; ++q) {
                if (how != SMALL) bytes += shapes[q]->x_bytes();
                most = imax(most, shapes[q]->matrices);
            }
            int64_t parts = imin(most, cdiv(bytes, MOST_X));
            for (int64_t part = 0; part < parts; ++part)
                if (!fill_batch(tensors, shapes, n, part, parts, &b)) {
                    if (parts >= most) return MOE_ERR_UNSUPPORTED;
                    parts = imin(most, 2 * parts);
                    part = -1;
                }
            for (int64_t part = 0; part < parts; ++part) {
                fill_batch(tensors, shapes, n, part, parts, &b);
                if (b.n) MOE_TRY(run(b, (How)how));
            }
        }
    return MOE_OK;
} catch (...) {
    return MOE_ERR_WORKSPACE;
}
struct Scratch {
    int32_t *done, *next;
    double *part;
    void *products;
};
int64_t blocks_of(const MuonBatch &b, bool second) {
    const MuonShape &s = b.s[b.shapes - 1];
    return second ? s.blocks_before + (int64_t)s.matrices * s.blocks : s.chunks_before + (int64_t)s.matrices * s.chunks;
}
Scratch scratch_of(Carver &cv, MuonBatch &b, bool pair) {
    Scratch s;
    s.next = cv.take<int32_t>(1);
    s.done = cv.take<int32_t>(b.matrices());
    s.part = cv.take<double>(blocks_of(b, false));
    for (int q = 0; q < b.shapes; ++q) b.s[q].x = cv.take<__half>((int64_t)b.s[q].matrices * b.s[q].rows * b.s[q].ld);
    s.products = cv.take_bytes(ns_scratch_bytes(b, pair));
    return s;
}

// Everything is made before the first launch: what is refused is refused before anything has changed
struct Ready {
    MuonBatch batch;
    How how;
    MuonPasses passes;
    NsLaunch products;
};

}  // namespace

int32_t muon_check(const moe_muon_tensor *tensors, int32_t count) {
    for (int32_t i = 0; i < count; ++i) MOE_TRY(check_tensor(tensors[i]));
    return MOE_OK;
}

int32_t muon_bytes(const moe_muon_tensor *tensors, int32_t count, int64_t *bytes) {
    *bytes = kWsHeader;
    return for_each_launch(tensors, count, [&](MuonBatch &b, How how) -> int32_t {
        if (how == SMALL) return MOE_OK;
        Carver cv(nullptr);
        cv.take_bytes(kWsHeader);
        scratch_of(cv, b, how == PAIRS);
        *bytes = imax(*bytes, (int64_t)cv.off);
        return MOE_OK;
    });
}

int32_t launch_muon(const moe_muon_tensor *tensors, int32_t count, const moe_muon_params &p, const moe_muon_rates *rates, void *ws, cudaStream_t st) {
    std::vector<std::unique_ptr<Ready>> all;
    MOE_TRY(for_each_launch(tensors, count, [&](MuonBatch &b, How how) -> int32_t {
        const bool pair = how == PAIRS;
        Carver cv(ws);
        int32_t *status = static_cast<int32_t *>(cv.take_bytes(kWsHeader));
        MuonPasses k = {};
        k.status = status;
        k.clear_status = all.empty(); k.nesterov = p.nesterov;
        k.momentum = (float)p.momentum; k.eps = (float)p.eps; k.grad_scale = (float)p.grad_scale; k.rates = rates;
        all.push_back(std::unique_ptr<Ready>(new Ready));
        Ready &r = *all.back();
        r.how = how;
        if (how == SMALL) {
            MOE_TRY(muon_small_ready());
        } else {
            const Scratch s = scratch_of(cv, b, pair);
            k.part = s.part; k.done = s.done; k.next = s.next;
            const NsWork w = {&b, pair, p.steps, s.done, s.next, status, s.products, (float)p.lr, rates};
            MOE_TRY(prepare_newton_schulz(w, &r.products));
        }
        r.batch = b;
        r.passes = k;
        return MOE_OK;
    }));
    for (const auto &one : all) {
        const MuonBatch &b = one->batch;
        const MuonPasses &k = one->passes;
        if (one->how == SMALL) {
            MOE_TRY(launch_muon_small(b, k, (float)p.lr, p.steps, st));
            continue;
        }
        launch_kernel(muon_momentum_kernel, dim3((unsigned)blocks_of(b, false)), dim3(THREADS), 0, st, b, k);
        MOE_LAUNCHED();
        launch_kernel(muon_normalise_kernel, dim3((unsigned)blocks_of(b, true)), dim3(THREADS), 0, st, b, k);
        MOE_LAUNCHED();
        MOE_TRY(launch_newton_schulz(one->products, b, st));
    }
    return MOE_OK;
}

}  // namespace moe
