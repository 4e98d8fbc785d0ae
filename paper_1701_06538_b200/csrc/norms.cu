// The norms around the block, one pass over memory each way.
//   norm_in:   xn = x r w,                              r  = (mean x^2 + eps)^-1/2
//   norm_out:  out = residual_scale x + gate (y r w),   r  = (mean y^2 + eps)^-1/2
//              next = out r2 w_next,                    r2 = (mean out^2 + eps)^-1/2   (the norm before the next block)
// Backward, with n = y r and n2 = out r2:
//   dt = dOut + r2 (dNext w_next - n2 mean(dNext w_next n2)),   dX = residual_scale dt,   dw_next = sum of dNext n2
//   dY = r (dt gate w - n mean(dt gate w n)),   dgate = w times the sum of dt n over the rows of the gate,   dw = sum of dt gate n
// All of it is bound by memory: a row stays in registers between its sums and what is made of it. Sums are float, over rows first by
// threads that keep their columns, then in double over what blocks have left, in a fixed order.
#include "block.cuh"

namespace moe {

namespace {

template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T *>(&raw)[i]); }
    __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T *>(&raw)[i] = from_f32<T>(v); }
};
template <typename T> __device__ __forceinline__ Vec<T> load_vec(const void *base, int64_t row, int32_t d, int32_t q) {
    Vec<T> v;
    v.raw = *reinterpret_cast<const uint4 *>(static_cast<const T *>(base) + row * d + (int64_t)q * Vec<T>::N);
    return v;
}
template <typename T> __device__ __forceinline__ void store_vec(void *base, int64_t row, int32_t d, int32_t q, const Vec<T> &v) {
    *reinterpret_cast<uint4 *>(static_cast<T *>(base) + row * d + (int64_t)q * Vec<T>::N) = v.raw;
}
template <int N> __device__ __forceinline__ void load_floats(const float *p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 a = *reinterpret_cast<const float4 *>(p + i);
        v[i] = a.x; v[i + 1] = a.y; v[i + 2] = a.z; v[i + 3] = a.w;
    }
}

// A row belongs to a team of `warps` warps of the block. Sums over the team's threads; `sh` has a place per team, warp and sum, twice, so that one
// barrier a row is enough: who writes the next row's sums does so on the other side, and the barrier of that row keeps it from coming round.
constexpr int MAX_SUMS = 4;
template <int K> __device__ __forceinline__ void team_sums(float (&s)[K], int warps, float *sh, int &side) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int i = 0; i < K; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], off);
    if (warps == 1) return;
    const int warp = threadIdx.x >> 5, team = warp / warps, lane = threadIdx.x & 31;
    float *mine = sh + side * (32 * MAX_SUMS);
    side ^= 1;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < K; ++i) mine[warp * MAX_SUMS + i] = s[i];
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory");
#pragma unroll
    for (int i = 0; i < K; ++i) s[i] = 0.0f;
    for (int q = 0; q < warps; ++q)
#pragma unroll
        for (int i = 0; i < K; ++i) s[i] += mine[(team * warps + q) * MAX_SUMS + i];
}

// Y: the block's output goes through its norm and the gate onto x; NEXT: a norm of the result (without Y: of x)
template <typename T, int V, bool Y, bool NEXT>
__global__ void __launch_bounds__(512) norm_rows_kernel(const NormArgs a, int warps) {
    wait_previous_kernel();
    constexpr int N = Vec<T>::N;
    __shared__ float sh[2 * 32 * MAX_SUMS];
    int side = 0;
    const int threads = warps * 32, teams = blockDim.x / threads, lane = threadIdx.x % threads;
    const int64_t row = (int64_t)blockIdx.x * teams + threadIdx.x / threads;
    if (row >= a.T) return;  // the whole team
    const int32_t pieces = a.d / N;
    const float by = 1.0f / (float)a.d;
    Vec<T> xv[V], yv[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int32_t q = lane + v * threads;
        if (q >= pieces) break;
        if constexpr (Y) yv[v] = load_vec<T>(a.y, row, a.d, q);
        xv[v] = load_vec<T>(a.x, row, a.d, q);
    }
    float o[V][N];
    float sum[1] = {0.0f};
    if constexpr (Y) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (lane + v * threads < pieces)
#pragma unroll
                for (int i = 0; i < N; ++i) { const float f = yv[v].get(i); sum[0] = fmaf(f, f, sum[0]); }
        team_sums(sum, warps, sh, side);
        const float r = 1.0f / sqrtf(sum[0] * by + a.eps);
        if (lane == 0) a.rstd[row] = r;
        const int64_t gate_row = a.gate ? (int64_t)((uint32_t)row / (uint32_t)a.rows_per_gate) : 0;
        sum[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            float w[N];
            load_floats(a.w + (int64_t)q * N, w);
            Vec<T> g, res;
            if (a.gate) g = load_vec<T>(a.gate, gate_row, a.d, q);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float u = yv[v].get(i) * r * w[i];
                if (a.gate) u *= g.get(i);
                o[v][i] = fmaf(a.residual_scale, xv[v].get(i), u);
                sum[0] = fmaf(o[v][i], o[v][i], sum[0]);
                res.set(i, o[v][i]);
            }
            store_vec<T>(a.out, row, a.d, q, res);
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (lane + v * threads < pieces)
#pragma unroll
                for (int i = 0; i < N; ++i) { o[v][i] = xv[v].get(i); sum[0] = fmaf(o[v][i], o[v][i], sum[0]); }
    }
    if constexpr (NEXT) {  // of what was not rounded yet
        team_sums(sum, warps, sh, side);
        const float r = 1.0f / sqrtf(sum[0] * by + a.eps);
        if (lane == 0 && a.rstd_next) a.rstd_next[row] = r;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            float w[N];
            load_floats(a.w_next + (int64_t)q * N, w);
            Vec<T> res;
#pragma unroll
            for (int i = 0; i < N; ++i) res.set(i, o[v][i] * r * w[i]);
            store_vec<T>(a.next, row, a.d, q, res);
        }
    }
}

// How the backward pass shares out its rows. With one gate (or none) a block has `rows` rows of one group and leaves partial sums (chunks of a
// group: `chunks`); with groups of a few rows a team has whole groups and writes their gate's gradient itself (chunks 0).
struct Share {
    int warps, teams, V;
    int64_t group, groups, chunks, rows, per_team, blocks;  // per_team: groups a team takes (chunks == 0)
};
constexpr int TEAM_ROWS = 4;
int64_t team_rows(int64_t T, int teams) { return imax(TEAM_ROWS, cdiv(T, (int64_t)teams * 148 * 6)); }
void team_of(int32_t d, int32_t act, int *warps, int *teams, int *V) {
    const int64_t pieces = d / (16 / (int64_t)act_bytes(act));
    *V = pieces <= 32 ? 1 : pieces <= 1024 ? 2 : pieces <= 2048 ? 4 : 8;  // at most 512 threads
    int w = 1;
    while (w * 32 * *V < pieces) w *= 2;
    *warps = w;
    *teams = w >= 8 ? 1 : 8 / w;
}
Share share_of(int64_t T, int32_t d, int32_t act, int64_t rows_per_gate) {
    Share s = {};
    team_of(d, act, &s.warps, &s.teams, &s.V);
    const int64_t each = team_rows(T, s.teams);
    s.group = rows_per_gate > 0 ? imin(rows_per_gate, imax(T, 1)) : imax(T, 1);
    s.groups = cdiv(T, s.group);
    s.rows = each * s.teams;
    if (rows_per_gate > 0 && s.group <= 2 * each) {
        s.per_team = imax(1, each / s.group);
        s.blocks = cdiv(s.groups, s.per_team * s.teams);
    } else {
        s.chunks = cdiv(s.group, s.rows);
        s.blocks = s.groups * s.chunks;
    }
    return s;
}
// more blocks than any rows_per_gate gives: whole groups fill at least half of a block's rows, and beside the chunks of `rows` rows there is at most one
// that is not full for every group, of more than 2 * each rows
int64_t most_blocks(int64_t T, int teams) {
    const int64_t each = team_rows(T, teams);
    return 2 * cdiv(T, each * teams) + T / (2 * each) + 3;
}

template <typename T, int V, bool Y, bool NEXT, bool GATE>
__global__ void __launch_bounds__(V == 1 ? 256 : 512) norm_grads_kernel(const NormGradArgs a, const Share s, float *part_w, float *part_next, float *part_gate) {
    wait_previous_kernel();
    constexpr int N = Vec<T>::N;
    extern __shared__ float columns[];  // [teams][d], where a block has several teams
    __shared__ float sh[2 * 32 * MAX_SUMS];
    int side = 0;
    const int threads = s.warps * 32, team = threadIdx.x / threads, lane = threadIdx.x % threads;
    const int32_t pieces = a.d / N;
    const float by = 1.0f / (float)a.d;
    float sum_n[V][N], sum_w[V][N], sum_next[V][N];  // of dt n over the group's rows so far; of dt gate n; of dNext n2
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < N; ++i) sum_n[v][i] = sum_w[v][i] = sum_next[v][i] = 0.0f;

    auto one_row = [&](int64_t row, int64_t gate_row) {
        Vec<T> dov[V], dnv[V], ov[V], yv[V], gv[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            if (a.dOut) dov[v] = load_vec<T>(a.dOut, row, a.d, q);
            else dov[v].raw = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (NEXT) {
                dnv[v] = load_vec<T>(a.dNext, row, a.d, q);
                ov[v] = load_vec<T>(a.out, row, a.d, q);
            }
            if constexpr (Y) yv[v] = load_vec<T>(a.y, row, a.d, q);
            if constexpr (GATE) gv[v] = load_vec<T>(a.gate, gate_row, a.d, q);
        }
        const float r = Y ? a.rstd[row] : 0.0f, r2 = NEXT ? a.rstd_next[row] : 0.0f;
        // c2 = mean(dn2 n2) decides dt, and c1 = mean(dt b) with b = gate w n the rest. Both are sums of one look at the row, since c1 is linear in dt:
        // mean(dOut b) + r2 (mean(dn2 b) - c2 mean(n2 b))
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            float w[N], wn[N];
            if constexpr (Y) load_floats(a.w + (int64_t)q * N, w);
            if constexpr (NEXT) load_floats(a.w_next + (int64_t)q * N, wn);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float b = 0.0f;
                if constexpr (Y) {
                    b = yv[v].get(i) * r * w[i];
                    if constexpr (GATE) b *= gv[v].get(i);
                    sum[1] = fmaf(dov[v].get(i), b, sum[1]);
                }
                if constexpr (NEXT) {
                    const float n2 = ov[v].get(i) * r2, dn2 = dnv[v].get(i) * wn[i];
                    sum[0] = fmaf(dn2, n2, sum[0]);
                    if constexpr (Y) {
                        sum[2] = fmaf(dn2, b, sum[2]);
                        sum[3] = fmaf(n2, b, sum[3]);
                    }
                }
            }
        }
        if constexpr (Y && NEXT) team_sums(sum, s.warps, sh, side);
        else {
            float one[1] = {sum[Y ? 1 : 0]};
            team_sums(one, s.warps, sh, side);
            sum[Y ? 1 : 0] = one[0];
        }
        const float c2 = sum[0] * by, c1 = (sum[1] + r2 * (sum[2] - c2 * sum[3])) * by;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            float w[N], wn[N];
            if constexpr (Y) load_floats(a.w + (int64_t)q * N, w);
            if constexpr (NEXT) load_floats(a.w_next + (int64_t)q * N, wn);
            Vec<T> dx, dy;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float dt = dov[v].get(i);
                if constexpr (NEXT) {
                    const float n2 = ov[v].get(i) * r2, g2 = dnv[v].get(i);
                    dt = fmaf(r2, g2 * wn[i] - n2 * c2, dt);
                    sum_next[v][i] = fmaf(g2, n2, sum_next[v][i]);
                }
                dx.set(i, a.residual_scale * dt);
                if constexpr (Y) {
                    const float n = yv[v].get(i) * r;
                    float dn = dt * w[i];
                    if constexpr (GATE) dn *= gv[v].get(i);
                    dy.set(i, r * (dn - n * c1));
                    sum_n[v][i] = fmaf(dt, n, sum_n[v][i]);
                }
            }
            store_vec<T>(a.dX, row, a.d, q, dx);
            if constexpr (Y) store_vec<T>(a.dY, row, a.d, q, dy);
        }
    };
    // the end of a group: its gate's gradient, and the group's part of dw
    auto end_group = [&](int64_t gate_row, bool write) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            const Vec<T> g = load_vec<T>(a.gate, gate_row, a.d, q);
            float w[N];
            load_floats(a.w + (int64_t)q * N, w);
            Vec<T> dg;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum_w[v][i] = fmaf(g.get(i), sum_n[v][i], sum_w[v][i]);
                dg.set(i, w[i] * sum_n[v][i]);
            }
            if (write) {
                store_vec<T>(a.dgate, gate_row, a.d, q, dg);
#pragma unroll
                for (int i = 0; i < N; ++i) sum_n[v][i] = 0.0f;
            }
        }
    };
    // the block's sums of its teams' columns, in the order of the teams. done(vector of columns, its sums)
    auto block_sums = [&](float (&mine)[V][N], auto done) {
        if (s.teams > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int32_t q = lane + v * threads;
                if (q >= pieces) break;
#pragma unroll
                for (int i = 0; i < N; i += 4)
                    *reinterpret_cast<float4 *>(columns + (int64_t)team * a.d + (int64_t)q * N + i) = make_float4(mine[v][i], mine[v][i + 1], mine[v][i + 2], mine[v][i + 3]);
            }
            __syncthreads();
            if (team > 0) return;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            float total[N];
#pragma unroll
            for (int i = 0; i < N; ++i) total[i] = mine[v][i];
            for (int t = 1; t < s.teams; ++t)
#pragma unroll
                for (int i = 0; i < N; ++i) total[i] += columns[(int64_t)t * a.d + (int64_t)q * N + i];
            done(q, total);
        }
    };
    auto to_part = [&](float *part) {
        return [=](int32_t q, const float (&total)[N]) {
#pragma unroll
            for (int i = 0; i < N; i += 4)
                *reinterpret_cast<float4 *>(part + (int64_t)blockIdx.x * a.d + (int64_t)q * N + i) = make_float4(total[i], total[i + 1], total[i + 2], total[i + 3]);
        };
    };

    if (GATE && s.chunks == 0) {
        const int64_t first = ((int64_t)blockIdx.x * s.teams + team) * s.per_team;
        for (int64_t g = first; g < min(first + s.per_team, s.groups); ++g) {
            const int64_t end = min((g + 1) * s.group, a.T);
            for (int64_t row = g * s.group; row < end; ++row) one_row(row, g);
            if constexpr (GATE) end_group(g, true);
        }
        if constexpr (Y && GATE) block_sums(sum_w, to_part(part_w));
    } else {
        const int64_t g = blockIdx.x / s.chunks, from = g * s.group + (blockIdx.x % s.chunks) * s.rows;
        const int64_t end = min(min(from + s.rows, (g + 1) * s.group), a.T);
        for (int64_t row = from + team; row < end; row += s.teams) one_row(row, g);
        if constexpr (Y && GATE) {
            end_group(g, false);
            block_sums(sum_w, to_part(part_w));
            if (s.chunks > 1) block_sums(sum_n, to_part(part_gate));
            else
                block_sums(sum_n, [&](int32_t q, const float (&total)[N]) {
                    float w[N];
                    load_floats(a.w + (int64_t)q * N, w);
                    Vec<T> dg;
#pragma unroll
                    for (int i = 0; i < N; ++i) dg.set(i, w[i] * total[i]);
                    store_vec<T>(a.dgate, g, a.d, q, dg);
                });
        } else if constexpr (Y) {
            block_sums(sum_n, to_part(part_w));
        }
    }
    if constexpr (NEXT) block_sums(sum_next, to_part(part_next));
}

// The blocks' sums added up, 32 columns a block, eight runs of blocks side by side, in double. Blocks of the grid: those of dw, of dw_next, then of every
// gate that several blocks share.
template <typename T>
__global__ void __launch_bounds__(256) norm_sums_kernel(const NormGradArgs a, const Share s, const float *part_w, const float *part_next, const float *part_gate) {
    wait_previous_kernel();
    __shared__ double sh[8][32];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int32_t slabs = (a.d + 31) / 32;
    const int64_t job = blockIdx.x / slabs;
    const int32_t col = (blockIdx.x % slabs) * 32 + lane;
    const float *part = nullptr;
    int64_t from = 0, count = s.blocks, gate_row = -1;
    float *to = nullptr;
    if (a.y && job == 0) { part = part_w; to = a.dw; }
    else if (a.dNext && job == (a.y ? 1 : 0)) { part = part_next; to = a.dw_next; }
    else {
        gate_row = job - (a.y ? 1 : 0) - (a.dNext ? 1 : 0);
        part = part_gate;
        from = gate_row * s.chunks;
        count = s.chunks;
    }
    const int64_t each = (count + 7) / 8, lo = from + run * each, hi = min(lo + each, from + count);
    double sum = 0.0;
    if (col < a.d) {
        float f[4];
        int64_t b = lo;
        for (; b + 4 <= hi; b += 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = part[(b + i) * a.d + col];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += f[i];
        }
        for (; b < hi; ++b) sum += part[b * a.d + col];
    }
    sh[run][lane] = sum;
    __syncthreads();
    if (run > 0 || col >= a.d) return;
    for (int i = 1; i < 8; ++i) sum += sh[i][lane];
    if (to) to[col] = (float)sum;
    else static_cast<T *>(a.dgate)[gate_row * a.d + col] = from_f32<T>((float)(a.w[col] * sum));
}

template <typename T, int V> int32_t launch_rows(const NormArgs &a, int warps, int teams, cudaStream_t st) {
    const dim3 grid((unsigned)cdiv(a.T, teams)), block(warps * 32 * teams);
    if (a.y && a.next) launch_kernel(norm_rows_kernel<T, V, true, true>, grid, block, 0, st, a, warps);
    else if (a.y) launch_kernel(norm_rows_kernel<T, V, true, false>, grid, block, 0, st, a, warps);
    else launch_kernel(norm_rows_kernel<T, V, false, true>, grid, block, 0, st, a, warps);
    MOE_LAUNCHED();
    return MOE_OK;
}

template <typename T, int V> int32_t launch_grads(const NormGradArgs &a, const Share &s, cudaStream_t st) {
    const int64_t most = most_blocks(a.T, s.teams) * a.d;
    float *part_w = a.ws, *part_next = part_w + most, *part_gate = part_next + most;
    if (s.blocks > 0) {
        const dim3 grid((unsigned)s.blocks), block(s.warps * 32 * s.teams);
        const size_t shared = s.teams > 1 ? sizeof(float) * s.teams * a.d : 0;
#define MOE_NORM_GRADS(Y, NEXT, GATE) launch_kernel(norm_grads_kernel<T, V, Y, NEXT, GATE>, grid, block, shared, st, a, s, part_w, part_next, part_gate)
        if (a.y && a.dNext && a.gate) MOE_NORM_GRADS(true, true, true);
        else if (a.y && a.dNext) MOE_NORM_GRADS(true, true, false);
        else if (a.y && a.gate) MOE_NORM_GRADS(true, false, true);
        else if (a.y) MOE_NORM_GRADS(true, false, false);
        else MOE_NORM_GRADS(false, true, false);
#undef MOE_NORM_GRADS
        MOE_LAUNCHED();
    }
    const int64_t jobs = (a.y ? 1 : 0) + (a.dNext ? 1 : 0) + (a.gate && s.chunks > 1 ? s.groups : 0);
    launch_kernel(norm_sums_kernel<T>, dim3((unsigned)(jobs * cdiv(a.d, 32))), dim3(256), 0, st, a, s, (const float *)part_w, (const float *)part_next, (const float *)part_gate);
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace

int64_t norm_grad_floats(int64_t T, int32_t d, int32_t act) {
    int warps, teams, V;
    team_of(d, act, &warps, &teams, &V);
    return 3 * most_blocks(T, teams) * d;
}

int32_t launch_norms(const NormArgs &a, cudaStream_t st) {
    if (a.T == 0) return MOE_OK;
    int warps, teams, V;
    team_of(a.d, a.act, &warps, &teams, &V);
    if (a.act == MOE_BF16) return V == 1 ? launch_rows<bf16, 1>(a, warps, teams, st) : V == 2 ? launch_rows<bf16, 2>(a, warps, teams, st) : launch_rows<bf16, 4>(a, warps, teams, st);
    return V == 1 ? launch_rows<float, 1>(a, warps, teams, st) : V == 2 ? launch_rows<float, 2>(a, warps, teams, st) : V == 4 ? launch_rows<float, 4>(a, warps, teams, st) : launch_rows<float, 8>(a, warps, teams, st);
}

int32_t launch_norm_grads(const NormGradArgs &a, cudaStream_t st) {
    const Share s = share_of(a.T, a.d, a.act, a.gate ? a.rows_per_gate : 0);
    if (a.act == MOE_BF16) return s.V == 1 ? launch_grads<bf16, 1>(a, s, st) : s.V == 2 ? launch_grads<bf16, 2>(a, s, st) : launch_grads<bf16, 4>(a, s, st);
    return s.V == 1 ? launch_grads<float, 1>(a, s, st) : s.V == 2 ? launch_grads<float, 2>(a, s, st) : s.V == 4 ? launch_grads<float, 4>(a, s, st) : launch_grads<float, 8>(a, s, st);
}

}  // namespace moe
